"""Refusals of the daf_page_* calls: everything that the host can see is refused before a launch, without a GPU."""
import ctypes

import pytest
import torch

from paper_2607_21599_b200 import api, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return api.lib()


def _params(**kw):
    a = dict(n_pages=10, page_tokens=32, n_kv_heads=2, n_seqs=4, max_pages=5, n_layers=3)
    a.update(kw)
    return api.make_page_params(**a)


def _buf(n=4096):
    b = torch.zeros(n + 16, dtype=torch.uint8)
    assert b.data_ptr() % 16 == 0
    return b


def test_struct_layout_matches_header():
    assert ctypes.sizeof(api.daf_page_params) == 28
    assert api.daf_page_params.max_pages.offset == 24


BAD = [(dict(n_pages=0), api.DAF_ERR_INVALID_ARG), (dict(n_pages=-3), api.DAF_ERR_INVALID_ARG),
       (dict(page_tokens=48), api.DAF_ERR_UNSUPPORTED), (dict(page_tokens=0), api.DAF_ERR_UNSUPPORTED),
       (dict(page_tokens=256), api.DAF_ERR_UNSUPPORTED), (dict(n_kv_heads=0), api.DAF_ERR_INVALID_ARG),
       (dict(n_kv_heads=257), api.DAF_ERR_UNSUPPORTED), (dict(head_dim=64), api.DAF_ERR_UNSUPPORTED),
       (dict(n_layers=0), api.DAF_ERR_INVALID_ARG), (dict(n_seqs=0), api.DAF_ERR_INVALID_ARG),
       (dict(max_pages=0), api.DAF_ERR_INVALID_ARG), (dict(max_pages=(1 << 22) // 32 + 1), api.DAF_ERR_UNSUPPORTED),
       (dict(n_pages=1 << 26), api.DAF_ERR_UNSUPPORTED), (dict(n_seqs=(1 << 20) + 1), api.DAF_ERR_UNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD)
def test_every_call_refuses_bad_parameters(change, status):
    p, b = _params(**change), _buf(1 << 16)
    assert api.daf_page_workspace_bytes(p, 1, 1, 4) == 0
    pool = (b, b, b, b)
    assert api.daf_page_write(p, 0, 1, None, b, b, None, 1, b, b, b, None, *pool, b) == status
    assert api.daf_page_read(p, 0, 1, None, None, b, 1, b, *pool, b, b, b) == status
    assert api.daf_page_attn(p, 0, 1, None, b, 1, 4, 0.0, b, b, *pool, b, None, b) == status
    assert api.daf_page_fork(p, 1, b, b, b, b, 1, b, b, *pool, b) == status
    assert api.daf_page_free(p, 1, b, None, b, b, b) == status
    assert api.daf_page_compact(p, b, b, b, b, None, *pool, b) == status


def test_workspace_sizes():
    p = _params()
    plain = api.daf_page_workspace_bytes(p, 4)
    attn = api.daf_page_workspace_bytes(p, 4, 1, 4)
    assert 256 < plain <= attn
    assert api.daf_page_workspace_bytes(p, 0) > 0
    assert api.daf_page_workspace_bytes(p, -1) == 0
    assert api.daf_page_workspace_bytes(p, 1, 1, 5) == 0           # not a multiple of the KV heads
    assert api.daf_page_workspace_bytes(p, 5000, 1, 4) == 0        # more sequences than one call takes
    with pytest.raises(api.DafError):
        api.alloc_page_workspace(p, 1, 1, 5, device="cpu")


def _calls(p, b, ws):
    """Each call with good arguments, as a function of replaced ones."""
    pool = dict(k8=b, v8=b, k_scale=b, v_scale=b)

    def write(layer=0, n=1, lens=b, row_off=b, max_rows=1, k=b, v=b, table=b, workspace=ws, **kw):
        x = {**pool, **kw}
        return api.daf_page_write(p, layer, n, None, lens, row_off, None, max_rows, k, v, table, None, x["k8"], x["v8"],
                                  x["k_scale"], x["v_scale"], workspace)

    def read(layer=0, n=1, row_off=b, max_rows=1, k=b, v=b, table=b, workspace=ws, **kw):
        x = {**pool, **kw}
        return api.daf_page_read(p, layer, n, None, None, row_off, max_rows, table, x["k8"], x["v8"], x["k_scale"], x["v_scale"],
                                 k, v, workspace)

    def attn(layer=0, n=1, lens=b, L_q=1, heads=4, q=b, table=b, out=b, lse=None, workspace=ws, **kw):
        x = {**pool, **kw}
        return api.daf_page_attn(p, layer, n, None, lens, L_q, heads, 0.0, q, table, x["k8"], x["v8"], x["k_scale"], x["v_scale"],
                                 out, lse, workspace)

    def fork(n=1, src=b, dst=b, keep=b, want=b, table=b, refs=b, workspace=ws, **kw):
        x = {**pool, **kw}
        return api.daf_page_fork(p, n, src, dst, keep, want, 1, table, refs, x["k8"], x["v8"], x["k_scale"], x["v_scale"], workspace)

    def free(n=1, seqs=b, keep=None, table=b, refs=b, workspace=ws):
        return api.daf_page_free(p, n, seqs, keep, table, refs, workspace)

    def compact(table=b, refs=b, table_out=b, refs_out=b, workspace=ws, **kw):
        x = {**pool, **kw}
        return api.daf_page_compact(p, table, refs, table_out, refs_out, None, x["k8"], x["v8"], x["k_scale"], x["v_scale"], workspace)

    return dict(write=write, read=read, attn=attn, fork=fork, free=free, compact=compact)


NEEDED = [("write", "lens"), ("write", "row_off"), ("write", "k"), ("write", "v"), ("write", "table"), ("write", "k8"),
          ("write", "v8"), ("write", "k_scale"), ("write", "v_scale"), ("read", "row_off"), ("read", "table"), ("read", "k"),
          ("read", "v"), ("read", "k8"), ("read", "v_scale"), ("attn", "lens"), ("attn", "q"), ("attn", "table"), ("attn", "out"),
          ("attn", "k8"), ("attn", "v8"), ("attn", "k_scale"), ("fork", "src"), ("fork", "dst"), ("fork", "keep"),
          ("fork", "want"), ("fork", "table"), ("fork", "refs"), ("fork", "v8"), ("free", "seqs"), ("free", "table"),
          ("free", "refs"), ("compact", "table"), ("compact", "refs"), ("compact", "table_out"), ("compact", "refs_out"),
          ("compact", "k_scale")]


@pytest.mark.parametrize("call,name", NEEDED)
def test_a_missing_tensor_is_refused(call, name):
    p, b = _params(), _buf()
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    assert _calls(p, b, ws)[call](**{name: None}) == api.DAF_ERR_INVALID_ARG


MISALIGNED = [("write", "k", 8), ("write", "v", 2), ("write", "k8", 8), ("write", "v8", 1), ("write", "k_scale", 2),
              ("write", "lens", 1), ("write", "table", 2), ("read", "k", 8), ("read", "v8", 4), ("read", "row_off", 3),
              ("attn", "q", 8), ("attn", "out", 4), ("attn", "k8", 8), ("attn", "lse", 2), ("attn", "lens", 1), ("fork", "src", 2),
              ("fork", "refs", 1), ("fork", "k8", 8), ("free", "seqs", 2), ("free", "table", 1), ("compact", "refs_out", 2),
              ("compact", "v8", 8)]


@pytest.mark.parametrize("call,name,by", MISALIGNED)
def test_a_misaligned_tensor_is_refused(call, name, by):
    p, b = _params(), _buf()
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    assert _calls(p, b, ws)[call](**{name: b[by:]}) == api.DAF_ERR_ALIGNMENT


@pytest.mark.parametrize("call", ["write", "read", "attn", "fork", "free", "compact"])
def test_workspace_is_checked(call):
    p, b = _params(), _buf()
    c = _calls(p, b, None)[call]
    assert c(workspace=None) == api.DAF_ERR_WORKSPACE
    assert c(workspace=b[:128]) == api.DAF_ERR_WORKSPACE
    big = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    assert c(workspace=big[8:]) in (api.DAF_ERR_ALIGNMENT, api.DAF_ERR_WORKSPACE)
    if call in ("attn", "fork", "compact"):
        need = api.daf_page_workspace_bytes(p, 1, 1, 4) if call == "attn" else api.daf_page_workspace_bytes(p, 1 if call == "fork" else 0)
        assert c(workspace=_buf(need)[:need - 1]) == api.DAF_ERR_WORKSPACE


def test_counts_layers_and_heads_are_checked():
    p, b = _params(), _buf()
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 4, 8))
    c = _calls(p, b, ws)
    for call in ("write", "read", "attn"):
        assert c[call](layer=-1) == api.DAF_ERR_INVALID_ARG
        assert c[call](layer=3) == api.DAF_ERR_INVALID_ARG
        assert c[call](n=-1) == api.DAF_ERR_INVALID_ARG
    for call in ("write", "read"):
        assert c[call](max_rows=-1) == api.DAF_ERR_INVALID_ARG
    assert c["attn"](heads=0) == api.DAF_ERR_INVALID_ARG
    assert c["attn"](heads=5) == api.DAF_ERR_UNSUPPORTED
    assert c["attn"](heads=512) == api.DAF_ERR_UNSUPPORTED
    assert c["attn"](n=2049) == api.DAF_ERR_UNSUPPORTED
    assert c["attn"](n=2048, L_q=4000) == api.DAF_ERR_UNSUPPORTED
    assert c["attn"](L_q=-1) == api.DAF_ERR_INVALID_ARG
    assert c["fork"](n=-1) == api.DAF_ERR_INVALID_ARG
    assert c["fork"](n=5) == api.DAF_ERR_INVALID_ARG               # more items than rows: one would be named twice
    assert c["free"](n=-1) == api.DAF_ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["write", "read", "attn", "fork", "free", "compact"])
def test_another_device_than_the_current_one_is_refused(call, monkeypatch):
    p, b = _params(), _buf()
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="current device"):
        _calls(p, b, ws)[call]()


def test_more_keys_than_an_attention_call_counts_are_refused():
    p, b = _params(n_kv_heads=8, max_pages=(1 << 22) // 32), _buf()          # pages of 32 tokens: 4M tokens a sequence
    ws = _buf(api.daf_page_workspace_bytes(p, 1024, 1, 8))
    assert api.daf_page_workspace_bytes(p, 1025, 1, 8) == 0
    assert _calls(p, b, ws)["attn"](n=1025, heads=8) == api.DAF_ERR_UNSUPPORTED


def test_nothing_to_do_is_ok_and_launches_nothing():
    p, b = _params(), _buf()
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    c = _calls(p, b, ws)
    before = api.daf_launch_count()
    for call in ("write", "read", "attn", "fork", "free"):
        assert c[call](n=0) == api.DAF_OK
    assert c["write"](max_rows=0) == api.DAF_OK and c["read"](max_rows=0) == api.DAF_OK and c["attn"](L_q=0) == api.DAF_OK
    assert api.daf_launch_count() == before


def test_status_text():
    assert "free pages" in api.daf_strerror(api.DAF_ERR_PAGES)


INTS, ROWS, BYTES, FLOATS = "int32", "bfloat16", "float8_e4m3fn", "reads torch.float32 elements"
READ_AS = [("write", n, t) for n, t in (("lens", INTS), ("row_off", INTS), ("table", INTS), ("k", ROWS), ("v", ROWS), ("k8", BYTES), ("v8", BYTES),
                                        ("k_scale", FLOATS), ("v_scale", FLOATS))]
READ_AS += [("read", n, t) for n, t in (("row_off", INTS), ("table", INTS), ("k", ROWS), ("v", ROWS), ("v8", BYTES), ("k_scale", FLOATS))]
READ_AS += [("attn", n, t) for n, t in (("lens", INTS), ("table", INTS), ("q", ROWS), ("out", ROWS), ("k8", BYTES), ("v_scale", FLOATS))]
READ_AS += [("fork", n, t) for n, t in (("src", INTS), ("dst", INTS), ("keep", INTS), ("want", INTS), ("table", INTS), ("refs", INTS), ("v8", BYTES), ("k_scale", FLOATS))]
READ_AS += [("free", n, INTS) for n in ("seqs", "table", "refs")]
READ_AS += [("compact", n, t) for n, t in (("table", INTS), ("refs", INTS), ("table_out", INTS), ("refs_out", INTS), ("k8", BYTES), ("v_scale", FLOATS))]
WRONG = {INTS: (torch.int64, torch.float32, torch.int16), ROWS: (torch.float32, torch.float16), BYTES: (torch.bfloat16, torch.float8_e5m2),
         FLOATS: (torch.float64, torch.bfloat16, torch.int32)}
RIGHT = {INTS: torch.int32, ROWS: torch.bfloat16, BYTES: torch.float8_e4m3fn, FLOATS: torch.float32}


@pytest.mark.parametrize("call,name,kind", READ_AS)
def test_tensors_of_other_types_are_refused(call, name, kind):
    """(n is 0 for those that are taken: nothing is launched.)"""
    p, b = _params(), _buf(1 << 16)
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    c = _calls(p, b, ws)[call]
    for t in WRONG[kind]:
        with pytest.raises(ValueError, match=kind):
            c(**{name: b[:1024].view(t)})
    if call != "compact":
        assert c(n=0, **{name: b[:1024].view(RIGHT[kind])}) == api.DAF_OK


@pytest.mark.parametrize("call,name,kind", READ_AS)
def test_each_tensor_has_to_be_on_the_current_device(call, name, kind, monkeypatch):
    p, b = _params(), _buf(1 << 16)
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)       # (where CPU tensors say that they are)
    elsewhere = _buf(1 << 16)
    monkeypatch.setattr(api, "_get_device", lambda t: 1 if t is elsewhere else -1)
    c = _calls(p, b, ws)[call]
    if call != "compact":
        monkeypatch.setattr(api, "_raw_stream", lambda device: 0)
        assert c(n=0) == api.DAF_OK
    for which in (name, "workspace"):
        with pytest.raises(ValueError, match="current device"):
            c(**{which: elsewhere})


def test_tensors_that_may_be_left_out_are_checked_as_well():
    p, b = _params(), _buf(1 << 16)
    ws = _buf(api.daf_page_workspace_bytes(p, 4, 1, 4))
    pool, w = (b, b, b, b), b[:64].view(torch.int64)
    for call in (lambda: api.daf_page_write(p, 0, 0, w, b, b, None, 1, b, b, b, None, *pool, ws),
                 lambda: api.daf_page_write(p, 0, 0, None, b, b, w, 1, b, b, b, None, *pool, ws),
                 lambda: api.daf_page_write(p, 0, 0, None, b, b, None, 1, b, b, b, w, *pool, ws),
                 lambda: api.daf_page_read(p, 0, 0, w, None, b, 1, b, *pool, b, b, ws),
                 lambda: api.daf_page_read(p, 0, 0, None, w, b, 1, b, *pool, b, b, ws),
                 lambda: api.daf_page_attn(p, 0, 0, w, b, 1, 4, 0.0, b, b, *pool, b, None, ws),
                 lambda: api.daf_page_attn(p, 0, 0, None, b, 1, 4, 0.0, b, b, *pool, b, w, ws),
                 lambda: api.daf_page_free(p, 0, b, w, b, b, ws),
                 lambda: api.daf_page_compact(p, b, b, b, b, w, *pool, ws)):
        with pytest.raises(ValueError, match="int64"):
            call()
