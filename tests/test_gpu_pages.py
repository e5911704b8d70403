"""The paged 8-bit cache on the GPU against its fp64 oracle: bytes, scales, tables and counts exactly, attention within a bound
derived from its roundings."""
import math
import random

import numpy as np
import pytest
import torch

from oracle import page_oracle as O
from paper_2607_21599_b200 import api, build

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """A pool with its table on the GPU, and the same in numpy."""

    def __init__(self, n_pages, T, Hkv, n_seqs, max_pages, n_layers=1, seed=0, junk=True, scale_exps=(-8, -4)):
        self.p = api.make_page_params(n_pages, T, Hkv, n_seqs, max_pages, n_layers=n_layers)
        self.T, self.Hkv, self.n_pages = T, Hkv, n_pages
        rng = np.random.default_rng(seed)
        shape = (n_layers, n_pages, Hkv, T, 128)
        # any bytes (NaN among them where junk): what nobody wrote must not matter
        self.np = {x + "8": rng.integers(0, 256, shape, dtype=np.uint8) for x in "kv"}
        if not junk:
            for x in "kv":
                a = self.np[x + "8"]
                a[(a & 127) == 127] ^= 1
        for x in "kv":
            self.np[x + "_scale"] = (2.0 ** rng.integers(scale_exps[0], scale_exps[1], shape[:3])).astype(np.float32)
        self.np["table"], self.np["refs"] = np.full((n_seqs, max_pages), -1, np.int32), np.zeros(n_pages, np.int32)
        self.order = rng.permutation(n_pages).tolist()
        self.up()

    def up(self):
        self.t = {n: torch.from_numpy(a.copy()).to(DEV) for n, a in self.np.items()}

    def give(self, seq, tokens, up=True):
        m = -(-tokens // self.T)
        for j in range(m):
            pg = self.order.pop()
            self.np["table"][seq, j] = pg
            self.np["refs"][pg] = 1
        if up:
            self.up()

    def pool(self):
        return self.t["k8"], self.t["v8"], self.t["k_scale"], self.t["v_scale"]

    def same(self, names=("k8", "v8", "k_scale", "v_scale", "table", "refs")):
        for n in names:
            got, want = self.t[n].cpu().numpy(), self.np[n]
            if n in ("k8", "v8"):      # one NaN is as good as the other
                got, want = np.where((got & 127) == 127, 127, got), np.where((want & 127) == 127, 127, want)
            assert np.array_equal(got, want), (n, np.argwhere(got != want)[:5])


def _ws(c, n=1, L_q=0, Hq=0):
    return api.alloc_page_workspace(c.p, n, L_q, Hq)


def _rows(n, Hkv, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, Hkv, 128, generator=g) * torch.exp2(spread * torch.randn(n, Hkv, 1, generator=g))
    return x.to(torch.bfloat16)


def _write(c, lens, counts, idx=None, seqs=None, k=None, v=None, refs=True, seed=1, layer=0, max_rows=None, status=api.DAF_OK, spread=1.0):
    R = sum(counts)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    k = _rows(R, c.Hkv, seed, spread) if k is None else k
    v = _rows(R, c.Hkv, seed + 1, spread) if v is None else v
    ws = _ws(c)
    i = None if idx is None else _i32(idx)
    api.check(api.daf_page_write(c.p, layer, len(lens), None if seqs is None else _i32(seqs), _i32(lens), torch.from_numpy(off).to(DEV),
                                 i, max(counts) if max_rows is None else max_rows, k.to(DEV), v.to(DEV), c.t["table"],
                                 c.t["refs"] if refs else None, *c.pool(), ws))
    assert api.daf_poll_status(ws) == status
    for x, rows in (("k", k), ("v", v)):
        O.write(c.np[x + "8"], c.np[x + "_scale"], layer, seqs, lens, off, idx, rows.float().numpy(), c.np["table"],
                c.np["refs"] if refs else None)


# --------------------------------------------------------------------------------------------------------------------- write
@pytest.mark.parametrize("T", [16, 32, 64, 128])
@pytest.mark.parametrize("Hkv", [1, 4, 5])
def test_append_ragged(T, Hkv):
    lens, counts = [1, T, T + 1, 3 * T - 1, 2 * T + 5, 0, 7], [1, T, 1, 2 * T, T + 3, 0, 0]
    c = Cache(40, T, Hkv, 7, 4, n_layers=2, seed=T + Hkv)
    for s, L in enumerate(lens):
        c.give(s, L)
    _write(c, lens, counts, layer=1)
    c.same()


def test_append_token_by_token_scales_grow():
    c = Cache(4, 16, 2, 1, 3, seed=5)
    c.give(0, 40)
    for t in range(1, 41):
        x = _rows(1, 2, 50 + t, spread=4.0)
        _write(c, [t], [1], k=x, v=(-0.25 * x.float()).to(torch.bfloat16))
    c.same()


@pytest.mark.parametrize("T,L,every", [(16, 100, 1), (64, 333, 3), (128, 1000, 7), (32, 64, 40), (64, 20000, 5)])
def test_rows_replaced_in_place(T, L, every):
    pages = -(-L // T)
    c = Cache(pages + 3, T, 2, 2, pages + 2, seed=L, junk=False)
    c.give(1, L)
    idx = list(range(every // 2, L, every))
    _write(c, [L], [len(idx)], idx=idx, seqs=[1], spread=3.0)
    c.same()


def test_rows_at_equal_positions_and_entries_of_all_kinds():
    c = Cache(30, 16, 3, 5, 6, seed=9, junk=False)
    for s in range(5):
        c.give(s, 80)
    # the last of equal rows counts, runs longer than a page among them; an entry without rows
    idx = [0, 0, 1, 17, 17, 17, 79] + [33] * 40 + [5, 64]
    _write(c, [80, 80, 70, 80], [7, 40, 0, 2], idx=idx, seqs=[4, 0, 2, 3], spread=3.0)
    c.same()


def test_special_values_and_borders():
    T = 16
    c = Cache(12, T, 1, 1, 12, seed=2)
    c.give(0, 12 * T)
    x = torch.zeros(12 * T, 1, 128)
    x[0:T] = 0.0                                        # a page of zeros
    x[T, 0, 0] = math.inf
    x[T, 0, 1] = 3.0
    x[T + 1, 0, 5] = math.nan
    x[T + 2, 0, 6] = -math.inf
    x[2 * T:3 * T] = 448.0
    x[3 * T:4 * T] = 450.0
    x[4 * T:5 * T] = 2.0 ** -66                         # below what the least scale holds with full precision
    x[5 * T, 0, 0] = 3e38
    x[5 * T + 1, 0, 0] = 1.0
    x[6 * T, 0, 0] = 1e-39                              # a subnormal
    x[7 * T:8 * T] = math.nan
    x[8 * T:9 * T, 0, :] = torch.arange(128) * 3.4375   # many ties between neighbours
    x[9 * T:10 * T] = -0.0
    x[10 * T] = math.inf                                # nothing finite
    x = x.to(torch.bfloat16)
    _write(c, [12 * T], [12 * T], k=x, v=-x)
    c.same()


def test_old_scales_that_are_no_powers_of_two():
    c = Cache(3, 32, 2, 1, 2, seed=3, junk=False)
    c.give(0, 40)
    for x in "kv":
        c.np[x + "_scale"][:] = np.float32(0.3)
    c.up()
    _write(c, [40], [1], spread=0.1)
    c.same()


def test_many_rows_over_several_grid_rounds_and_small_max_rows():
    c = Cache(20, 16, 1, 1, 20, seed=4)
    c.give(0, 300)
    _write(c, [300], [290], max_rows=5)        # a hint that is too small costs time, not rows
    c.same()


@pytest.mark.parametrize("T", [16, 32])
def test_neighbouring_pages_are_written_apart(T):
    # neighbouring pages whose rows differ by many powers of two, one of them missing, one shared, a first and a last kept in part
    c = Cache(40, T, 2, 2, 9, seed=T, junk=False)
    for s in range(2):
        c.give(s, 9 * T)
    c.np["table"][0, 3] = -1
    c.np["refs"][c.np["table"][0, 5]] = 2
    c.up()
    L, R = 9 * T - 3, 8 * T + 1
    x = [(_rows(R, 2, seed, 0.0).float() * torch.exp2(-4.0 * (torch.arange(R) // 5 % 7).float())[:, None, None]).to(torch.bfloat16) for seed in (1, 2)]
    _write(c, [L], [R], k=x[0], v=x[1], status=api.DAF_ERR_BOUNDS)
    c.same()
    _write(c, [L, L - 4], [R, 3 * T], k=torch.cat([x[1], x[0][:3 * T]]), v=torch.cat([x[0], x[1][:3 * T]]), seqs=[1, 0], status=api.DAF_ERR_BOUNDS,
           max_rows=2 ** 31 - 1)
    c.same()


def test_write_skips_and_reports_what_is_out_of_range():
    c = Cache(20, 16, 2, 4, 4, seed=6)
    for s in range(4):
        c.give(s, 64)
    c.np["table"][0, 1] = -1
    c.np["table"][1, 0] = 20
    c.np["refs"][c.np["table"][2, 2]] = 2
    c.up()
    _write(c, [64, 64, 64, 64], [64, 64, 64, 64], status=api.DAF_ERR_BOUNDS)
    c.same()
    _write(c, [64, 64, 64, 64], [64, 64, 64, 64], status=api.DAF_ERR_BOUNDS, refs=False, seed=77)
    c.same()
    for lens, seqs in (([65], None), ([-1], None), ([10], [4]), ([10], [-1])):
        before = {n: t.clone() for n, t in c.t.items()}
        ws = _ws(c)
        x = _rows(12, 2, 1).to(DEV)
        api.check(api.daf_page_write(c.p, 0, 1, None if seqs is None else _i32(seqs), _i32(lens), _i32([0, 12]), None, 12, x, x,
                                     c.t["table"], None, *c.pool(), ws))
        assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
        for n, t in c.t.items():
            assert torch.equal(t, before[n]), n


def test_positions_outside_the_sequence_are_skipped():
    c = Cache(8, 16, 1, 1, 4, seed=8, junk=False)
    c.give(0, 64)
    ws = _ws(c)
    x = _rows(3, 1, 4)
    api.check(api.daf_page_write(c.p, 0, 1, None, _i32([40]), _i32([0, 3]), _i32([3, 39, 41]), 3, x.to(DEV), x.to(DEV), c.t["table"],
                                 c.t["refs"], *c.pool(), ws))
    assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
    for n in "kv":
        O.write(c.np[n + "8"], c.np[n + "_scale"], 0, None, [40], [0, 2], [3, 39], x[:2].float().numpy(), c.np["table"])
    c.same()


@pytest.mark.parametrize("length,idx,inside", [(64, [-1, 5, 9], [1, 2]), (20, [5, 48, 63], [0]), (20, [64, 65, 1000], []), (0, [0, 1, 2], [])])
def test_positions_far_outside_the_sequence_are_reported(length, idx, inside):
    c = Cache(8, 16, 1, 1, 4, seed=8, junk=False)
    c.give(0, 64)
    ws = _ws(c)
    x = _rows(3, 1, 4)
    api.check(api.daf_page_write(c.p, 0, 1, None, _i32([length]), _i32([0, 3]), _i32(idx), 3, x.to(DEV), x.to(DEV), c.t["table"],
                                 c.t["refs"], *c.pool(), ws))
    assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
    for n in "kv":
        O.write(c.np[n + "8"], c.np[n + "_scale"], 0, None, [length], [0, len(inside)], [idx[i] for i in inside], x[inside].float().numpy(), c.np["table"])
    c.same()


def test_rows_replaced_in_a_table_of_many_columns():
    # more columns than an entry has thread blocks: 2 * 8 heads * 4 entries leave each 256
    c = Cache(2100, 16, 8, 4, 1000, seed=12, junk=False)
    lens = [16000, 30, 9001, 5000]
    for s, L in enumerate(lens):
        c.give(s, L, up=False)
    c.up()
    idx = [list(range(s, L, 37 + s)) for s, L in enumerate(lens)]
    _write(c, lens, [len(i) for i in idx], idx=sum(idx, []), spread=3.0)
    c.same()


# ---------------------------------------------------------------------------------------------------------------------- read
@pytest.mark.parametrize("T,Hkv", [(16, 1), (32, 8), (64, 4), (128, 3)])
def test_read(T, Hkv):
    c = Cache(30, T, Hkv, 3, 9, n_layers=2, seed=T)
    for s, L in enumerate((9 * T, 1, 2 * T + 3)):
        c.give(s, L)
    first, counts, seqs = [3, 0, T, T - 1, 5], [8 * T - 3, 1, T + 3, 2, 0], [0, 1, 2, 0, 2]
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    R = int(off[-1])
    k = torch.full((R + 1, Hkv, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    ws = _ws(c)
    api.check(api.daf_page_read(c.p, 1, 5, _i32(seqs), _i32(first), _i32(off.tolist()), max(counts), c.t["table"], *c.pool(), k, v, ws))
    assert api.daf_poll_status(ws) == api.DAF_OK
    for x, got in (("k", k), ("v", v)):
        for b in range(5):
            want = O.read(c.np[x + "8"], c.np[x + "_scale"], 1, seqs[b], first[b], counts[b], c.np["table"])
            here = got[off[b]:off[b + 1]].float().cpu().numpy()
            assert np.array_equal(np.isnan(here), np.isnan(want)) and np.array_equal(np.nan_to_num(here), np.nan_to_num(want)), (x, b)
        assert torch.all(got[R] == 7.0), "a row behind the last was written"


def test_read_reports_missing_pages():
    MARK = 2.0 ** 99        # no byte is worth that here
    c = Cache(8, 16, 1, 2, 3, seed=1, junk=False)
    c.give(0, 48)
    c.np["table"][0, 1] = 8
    c.up()
    k = torch.full((48, 1, 128), MARK, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    ws = _ws(c)
    api.check(api.daf_page_read(c.p, 0, 1, None, None, _i32([0, 48]), 48, c.t["table"], *c.pool(), k, v, ws))
    assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
    assert torch.all(k[16:32] == MARK) and not torch.any(k[:16] == MARK) and not torch.any(v[32:] == MARK)
    for first, seq in (([1], [0]), ([-1], [0]), ([0], [2])):
        k.fill_(MARK)
        api.check(api.daf_page_read(c.p, 0, 1, _i32(seq), _i32(first), _i32([0, 48]), 48, c.t["table"], *c.pool(), k, v, ws))
        assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
        assert torch.all(k == MARK)


# ----------------------------------------------------------------------------------------------------------------- attention
def _attend(c, lens, L_q, Hq, seqs=None, q=None, layer=0, scale=0.0, status=api.DAF_OK, seed=0, check=True, missing=None, q_scale=1.0):
    """Runs daf_page_attn and holds it to the oracle.

    The bound, element by element: the output's rounding to bf16 is 2^-8 |o|; P's to fp16 is 2^-11 of each p, so 2^-11 sum p |v|;
    an error d in a logit changes p by d, where d <= 2^-17 sum |q| |k| scale (fp32 sums of 128 products on the tensor cores, at most
    64 roundings of 2^-23) + 2^-20 (three roundings of the exponent's argument for |z| < 2^2, the exponential's 2^-22), and p's
    normalisation by as much again; a step of fp16 below 2^-14 is 2^-24, and P's largest value is at least 2^9, so that P is off by
    2^-25 / 2^9 of the largest p vs however small it is: 2^-34 L 448 max(vs)."""
    n = len(lens)
    g = torch.Generator().manual_seed(seed + 100)
    q = (torch.randn(n, L_q, Hq, 128, generator=g) * q_scale).to(torch.bfloat16) if q is None else q
    out = torch.full((n + 1, L_q, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n + 1, Hq, L_q), 7.0, device=DEV)
    ws = _ws(c, n, L_q, Hq)
    ws[256:] = 0xFF                                        # what an earlier call left there must not matter
    api.check(api.daf_page_attn(c.p, layer, n, None if seqs is None else _i32(seqs), _i32(lens), L_q, Hq, scale, q.to(DEV), c.t["table"],
                                *c.pool(), out[:n], lse[:n], ws))
    assert api.daf_poll_status(ws) == status
    assert torch.all(out[n] == 7.0) and torch.all(lse[n] == 7.0), "rows behind the last sequence were written"
    got, got_lse = out[:n].float().cpu().numpy().astype(np.float64), lse[:n].cpu().numpy().astype(np.float64)
    if not check:
        return got, got_lse
    sm = scale if scale > 0 else 1 / math.sqrt(128)
    for b in range(n):
        seq = b if seqs is None else seqs[b]
        L = max(0, lens[b])
        k = O.values(c.np["k8"], c.np["k_scale"], layer, seq, L, c.np["table"])
        v = O.values(c.np["v8"], c.np["v_scale"], layer, seq, L, c.np["table"])
        present = np.array([0 <= c.np["table"][seq, t // c.T] < c.n_pages for t in range(L)], bool)
        want, want_lse, mag, dots = O.attn(q[b].float().numpy().astype(np.float64), k, v, L, present, sm)
        d = 2.0 ** -17 * dots + 2.0 ** -20 + 2.0 ** -23 * np.abs(np.nan_to_num(want_lse, neginf=0.0).T)
        lost = 2.0 ** -34 * L * 448 * float(np.nanmax(c.np["v_scale"][layer]))
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2 * d[..., None]) * mag * 1.01 + lost
        assert np.array_equal(np.isnan(got[b]), np.isnan(want)), (b, np.argwhere(np.isnan(got[b]) != np.isnan(want))[:4])
        ok = (np.abs(got[b] - want) <= tol) | np.isnan(want)
        assert ok.all(), (b, np.argwhere(~ok)[:4], np.abs(got[b] - want)[~ok][:4], tol[~ok][:4])
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse[b]), empty) and not got[b].transpose(1, 0, 2)[empty].any()
        fine = ~empty & ~np.isnan(want_lse)
        err = np.abs(got_lse[b][fine] - want_lse[fine])
        assert (err <= (d.T + 2.0 ** -21 + 2.0 ** -22 * np.abs(want_lse))[fine]).all(), (b, err.max())
        assert np.array_equal(np.isnan(got_lse[b]), np.isnan(want_lse))
    return got, got_lse


def _cache_for(lens, T, Hkv, seed=0, n_layers=1, **kw):
    pages = [-(-max(0, L) // T) for L in lens]
    c = Cache(sum(pages) + 2, T, Hkv, len(lens), max(pages) + 1, n_layers=n_layers, seed=seed, **kw)
    for s, L in enumerate(lens):
        c.give(s, max(0, L), up=False)
    c.up()
    return c


HEADS = [(28, 4), (32, 8), (40, 8), (4, 4), (8, 1), (16, 1), (24, 1), (6, 2)]


@pytest.mark.parametrize("T", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_decode_lengths(T, Hq, Hkv):
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 0, 300, 517]
    c = _cache_for(lens, T, Hkv, seed=T * Hq, junk=False)
    _attend(c, lens, 1, Hq)


@pytest.mark.parametrize("L_q", [2, 3, 5, 17, 33, 70, 130])
@pytest.mark.parametrize("Hq,Hkv,T", [(28, 4, 64), (8, 2, 16), (5, 5, 32), (16, 1, 128)])
def test_several_query_tokens(L_q, Hq, Hkv, T):
    lens = [L_q, 1, 0, L_q - 1, L_q + 1, 200, 64, 3 * L_q + 31]
    c = _cache_for(lens, T, Hkv, seed=L_q, junk=False)
    _attend(c, lens, L_q, Hq)


@pytest.mark.parametrize("L_q", [1, 3, 40])
def test_bytes_behind_the_last_token_do_not_matter(L_q):
    lens = [5, 33, 70, 127, 1, 200]
    c = _cache_for(lens, 64, 2, seed=11, junk=False)
    for x in "kv":
        a = c.np[x + "8"]
        live = np.zeros(a.shape[1:4:2], bool)
        for s, L in enumerate(lens):
            for t in range(L):
                live[c.np["table"][s, t // 64], t % 64] = True
        a[0][~live[:, None, :].repeat(2, 1)] = 0x7F        # NaN wherever no token lies
        c.np[x + "_scale"][0, c.np["refs"] == 0] = np.nan
    c.up()
    _attend(c, lens, L_q, 8)


@pytest.mark.parametrize("L_q,Hq", [(4, 4), (6, 14), (40, 14)])
def test_nan_reaches_only_the_rows_that_see_it(L_q, Hq):
    lens = [20, 75, 130]
    c = _cache_for(lens, 32, 2, seed=12, junk=False)
    # a NaN in a value that the last tokens of the call see, in one that all see, and in a key of the last token
    def put(x, s, t, h, d):
        c.np[x][0, c.np["table"][s, t // 32], h, t % 32, d] = 0xFF
    put("v8", 0, 18, 0, 7)
    put("v8", 0, 19, 1, 127)
    put("v8", 1, 73, 0, 64)
    put("v8", 1, 10, 1, 3)
    put("k8", 2, 129, 0, 5)
    c.up()
    _attend(c, lens, L_q, Hq)


def test_all_keys_nan():
    c = _cache_for([40], 16, 1, seed=1, junk=False)
    c.np["k8"][:] = 0x7F
    c.up()
    got, lse = _attend(c, [40], 1, 2, check=False)
    assert np.isnan(got).all() and np.isnan(lse).all()


def test_scales_of_all_sizes():
    lens = [130, 77, 600]
    c = _cache_for(lens, 16, 2, seed=13, junk=False, scale_exps=(-30, -4))
    rng = np.random.default_rng(1)
    c.np["v_scale"][:] = (2.0 ** rng.integers(-40, 30, c.np["v_scale"].shape)).astype(np.float32)
    c.np["v_scale"][0, ::3] *= np.float32(1.37)            # a caller's own scales
    c.np["k_scale"][0, ::2] *= np.float32(0.7)
    c.up()
    for L_q in (1, 5, 50):
        _attend(c, lens, L_q, 6)


@pytest.mark.parametrize("L_q", [1, 30])
def test_sharp_and_flat_rows(L_q):
    lens = [500, 333]
    c = _cache_for(lens, 64, 2, seed=14, junk=False, scale_exps=(-7, -5))
    q = torch.randn(2, L_q, 8, 128, generator=torch.Generator().manual_seed(1))
    q[0, :, 0] *= 30.0                      # one key takes nearly all
    q[0, :, 1] = 0.0                        # all keys alike
    q[0, :, 2] *= 1e-30
    q[1, :, 3] *= 2.0 ** torch.linspace(-30, 3, 128)      # channels of very different size
    _attend(c, lens, L_q, 8, q=q.to(torch.bfloat16))
    _attend(c, lens, L_q, 8, scale=0.5, seed=3, q_scale=0.3)


def test_infinite_and_nan_queries_stay_in_their_rows():
    lens = [100]
    c = _cache_for(lens, 32, 1, seed=15, junk=False)
    for L_q in (1, 20):
        q = torch.randn(1, L_q, 4, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
        good, _ = _attend(c, lens, L_q, 4, q=q)
        q[0, 0, 1, 5] = math.inf
        q[0, 0, 2, 9] = math.nan
        got, _ = _attend(c, lens, L_q, 4, q=q, check=False)
        assert np.isnan(got[0, 0, 1:3]).all()
        assert np.array_equal(got[0, :, 0], good[0, :, 0]) and np.array_equal(got[0, :, 3], good[0, :, 3])
        assert np.array_equal(got[0, 1:], good[0, 1:])


@pytest.mark.parametrize("L_q", [1, 4, 24])
def test_missing_pages_count_as_absent_and_are_reported(L_q):
    lens = [100, 200, 40]
    c = _cache_for(lens, 16, 2, seed=16, junk=False)
    c.np["table"][0, 2] = -1
    c.np["table"][1, 0] = c.n_pages
    c.np["table"][1, 7:10] = -5
    c.np["table"][2, :] = -1
    c.up()
    _attend(c, lens, L_q, 8, status=api.DAF_ERR_BOUNDS)


@pytest.mark.parametrize("L_q", [1, 20])
def test_bad_lengths_and_rows_are_reported(L_q):
    c = _cache_for([100, 60], 16, 2, seed=17, junk=False)
    for lens, seqs in (([-4, 60], None), ([100, 60], [0, 2]), ([100, 60], [-1, 1])):
        got, lse = _attend(c, lens, L_q, 4, seqs=seqs, status=api.DAF_ERR_BOUNDS, check=False)
        for b in range(2):
            bad = lens[b] < 0 or (seqs is not None and not 0 <= seqs[b] < 2)
            assert np.isneginf(lse[b]).all() == bad and (not got[b].any()) == bad
    _attend(c, [10 ** 9, 60], L_q, 4, status=api.DAF_ERR_BOUNDS, check=False)      # longer than its row of the table


def test_rows_of_the_table_in_any_order_and_twice():
    lens = [64, 10, 200, 33]
    c = _cache_for(lens, 32, 2, seed=18, junk=False, n_layers=2)
    seqs = [2, 0, 2, 3, 1]
    for L_q in (1, 18):
        _attend(c, [200, 64, 150, 33, 10], L_q, 4, seqs=seqs, layer=1)


@pytest.mark.parametrize("n,L_q,Hq,Hkv", [(300, 1, 4, 2), (2048, 1, 1, 1), (150, 20, 4, 1)])
def test_many_sequences(n, L_q, Hq, Hkv):
    rng = random.Random(n)
    lens = [rng.randint(0, 60) for _ in range(n)]
    c = _cache_for(lens, 16, Hkv, seed=n, junk=False)
    if n < 1000:
        _attend(c, lens, L_q, Hq)
        return
    got, _ = _attend(c, lens, L_q, Hq, check=False)         # the oracle on a sample
    for b in range(0, n, 97):
        k = O.values(c.np["k8"], c.np["k_scale"], 0, b, lens[b], c.np["table"])
        v = O.values(c.np["v8"], c.np["v_scale"], 0, b, lens[b], c.np["table"])
        q = torch.randn(n, L_q, Hq, 128, generator=torch.Generator().manual_seed(100)).to(torch.bfloat16)[b]
        want, _, mag, dots = O.attn(q.float().numpy().astype(np.float64), k, v, lens[b])
        assert (np.abs(got[b] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -16 * dots[..., None] + 2.0 ** -18) * mag + 1e-9).all(), b


def _torch_attend(c, L, L_q, Hq, q, seq=0):
    """fp64 on the GPU, for lengths that the loops of the oracle are too slow for."""
    pages = c.t["table"][seq, :-(-L // c.T)].long()
    lut = torch.from_numpy(O.VALUES).to(DEV)
    k, v = [(lut[c.t[x + "8"][0][pages].long()] * c.t[x + "_scale"][0][pages].double()[..., None, None]).transpose(1, 2).reshape(-1, c.Hkv, 128)[:L] for x in "kv"]
    out = torch.zeros(L_q, Hq, 128, dtype=torch.float64, device=DEV)
    mag, dots = torch.zeros_like(out), torch.zeros(L_q, Hq, dtype=torch.float64, device=DEV)
    G = Hq // c.Hkv
    for h in range(Hq):
        kk, vv, qq = k[:, h // G], v[:, h // G], q[:, h].double().to(DEV)
        z = qq @ kk.T / math.sqrt(128)
        z = z.masked_fill(torch.arange(L, device=DEV)[None] > (L - L_q + torch.arange(L_q, device=DEV))[:, None], -math.inf)
        p = z.softmax(-1)
        out[:, h], mag[:, h] = p @ vv, p @ vv.abs()
        dots[:, h] = (qq.abs() @ kk.abs().T).amax(-1) / math.sqrt(128)
    return out, mag, dots


@pytest.mark.parametrize("L,L_q,Hq,Hkv,T", [(70001, 1, 7, 1, 64), (33000, 1, 28, 4, 16), (20011, 16, 8, 2, 128), (9000, 128, 28, 4, 64),
                                            (5000, 333, 8, 8, 32), (40000, 64, 16, 1, 16), (131, 131, 28, 4, 16), (3000, 1500, 4, 2, 64)])
def test_long_sequences(L, L_q, Hq, Hkv, T):
    c = _cache_for([L], T, Hkv, seed=L, junk=False, scale_exps=(-8, -6))
    q = torch.randn(1, L_q, Hq, 128, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    got, _ = _attend(c, [L], L_q, Hq, q=q, check=False)
    want, mag, dots = (x.cpu().numpy() for x in _torch_attend(c, L, L_q, Hq, q[0]))
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -16 * dots[..., None] + 2.0 ** -19) * mag * 1.01 + 2.0 ** -34 * L * 448 * 2.0 ** -6
    assert (np.abs(got[0] - want) <= tol).all(), np.abs(got[0] - want).max()


@pytest.mark.parametrize("L_q,Hq,Hkv", [(1, 256, 256), (26, 256, 256), (1, 256, 1), (3, 256, 1), (1, 200, 8), (2, 39, 3)])
def test_head_counts_at_the_limits(L_q, Hq, Hkv):
    lens = [70, 1, 200] if Hkv < 256 else [70, 33]
    c = _cache_for(lens, 32, Hkv, seed=Hq + L_q, junk=False)
    _attend(c, lens, L_q, Hq)


def test_a_question_of_every_sequence_of_a_full_call():
    n, L_q = 2048, 30
    rng = random.Random(3)
    lens = [rng.randint(0, 90) for _ in range(n)]
    c = _cache_for(lens, 16, 1, seed=31, junk=False, scale_exps=(-8, -6))
    q = torch.randn(n, L_q, 1, 128, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    got, _ = _attend(c, lens, L_q, 1, q=q, check=False)
    for b in range(0, n, 61):
        sees = max(0, L_q - lens[b])                 # rows in front of the first that sees a key
        assert not got[b, :sees].any()
        if lens[b] == 0:
            continue
        want, mag, dots = (x.cpu().numpy()[sees:] for x in _torch_attend(c, lens[b], L_q, 1, q[b], seq=b))
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -16 * dots[..., None] + 2.0 ** -19) * mag * 1.01 + 2.0 ** -34 * 90 * 448 * 2.0 ** -6
        assert (np.abs(got[b, sees:] - want) <= tol).all(), b


@pytest.mark.parametrize("L_q", [1, 30])
def test_a_sequence_of_millions_of_tokens(L_q):
    L, T = 2_000_003, 128
    c = _cache_for([L], T, 1, seed=7, junk=False, scale_exps=(-8, -6))
    q = torch.randn(1, L_q, 1, 128, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    got, _ = _attend(c, [L], L_q, 1, q=q, check=False)
    want, mag, dots = (x.cpu().numpy() for x in _torch_attend(c, L, L_q, 1, q[0]))
    # fp32 sums: L / 148 keys, 16 at a time, one behind the other, and 148 partial ones (2^-24 of the running sum each)
    sums = (L / 148 / 16 + 148) * 2.0 ** -24
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -16 * dots[..., None] + 2.0 ** -19 + sums) * mag * 1.01 + 2.0 ** -34 * L * 448 * 2.0 ** -6
    assert (np.abs(got[0] - want) <= tol).all(), np.abs(got[0] - want).max()


@pytest.mark.parametrize("L_q", [1, 40])
def test_pages_beyond_4_gb(L_q):
    """A layer of more than 2^32 bytes: the sequence's pages are the last ones."""
    T, Hkv, n_pages, L = 128, 8, 33000, 700
    assert n_pages * Hkv * T * 128 > 2 ** 32
    p = api.make_page_params(n_pages, T, Hkv, 1, 6)
    k8 = torch.empty(1, n_pages, Hkv, T, 128, dtype=torch.uint8, device=DEV)
    v8 = torch.empty_like(k8)
    ks, vs = torch.ones(1, n_pages, Hkv, device=DEV), torch.ones(1, n_pages, Hkv, device=DEV)
    table = torch.arange(n_pages - 6, n_pages, dtype=torch.int32, device=DEV).flip(0).contiguous().view(1, 6)
    refs = torch.ones(n_pages, dtype=torch.int32, device=DEV)
    ws = api.alloc_page_workspace(p, 1, L_q, 16)
    k, v = _rows(L, Hkv, 1, 0.0).to(DEV), _rows(L, Hkv, 2, 0.0).to(DEV)
    api.check(api.daf_page_write(p, 0, 1, None, _i32([L]), _i32([0, L]), None, L, k, v, table, refs, k8, v8, ks, vs, ws))
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    api.check(api.daf_page_read(p, 0, 1, None, None, _i32([0, L]), L, table, k8, v8, ks, vs, rk, rv, ws))
    # a byte is within 2^-4 of its value, or half a step of the smallest (2^-10 scales)
    for a, b in ((k, rk), (v, rv)):
        assert ((a.float() - b.float()).abs() <= a.float().abs() * 2.0 ** -4 + 2.0 ** -10 * 2.0 ** -6).all()
    q = torch.randn(1, L_q, 16, 128, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16)
    out = torch.empty(1, L_q, 16, 128, dtype=torch.bfloat16, device=DEV)
    api.check(api.daf_page_attn(p, 0, 1, None, _i32([L]), L_q, 16, 0.0, q.to(DEV), table, k8, v8, ks, vs, out, None, ws))
    assert api.daf_poll_status(ws) == api.DAF_OK
    mask = torch.arange(L, device=DEV)[None] > (L - L_q + torch.arange(L_q, device=DEV))[:, None]
    for h in range(16):
        z = (q[0, :, h].double().to(DEV) @ rk[:, h // 2].double().T / math.sqrt(128)).masked_fill(mask, -math.inf)
        pr = z.softmax(-1)
        want, mag = pr @ rv[:, h // 2].double(), pr @ rv[:, h // 2].double().abs()
        assert ((out[0, :, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * mag).all()


def test_results_do_not_depend_on_the_run():
    lens = [700, 3, 5000, 64, 1200]
    c = _cache_for(lens, 16, 4, seed=21, junk=False)
    for L_q in (1, 3, 30):
        a = _attend(c, lens, L_q, 28, check=False)
        for _ in range(3):
            b = _attend(c, lens, L_q, 28, check=False)
            assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


# ------------------------------------------------------------------------------------------------------------ pages of the pool
def _snapshot(c):
    return {n: a.copy() for n, a in c.np.items()}


def _pool(c):
    return O.Pool(c.np["table"], c.np["refs"], c.T, [c.np["k8"], c.np["v8"], c.np["k_scale"], c.np["v_scale"]])


def _fork(c, src, dst, keep, want, share, ws=None):
    said = _pool(c).fork(src, dst, keep, want, share)
    ws = _ws(c, len(src)) if ws is None else ws
    api.check(api.daf_page_fork(c.p, len(src), _i32(src), _i32(dst), _i32(keep), _i32(want), share, c.t["table"], c.t["refs"], *c.pool(), ws))
    assert api.daf_poll_status(ws) == {"": api.DAF_OK, "bounds": api.DAF_ERR_BOUNDS, "pages": api.DAF_ERR_PAGES}[said]
    c.same()
    return said


def _free(c, seqs, keep=None):
    _pool(c).free(seqs, keep)
    ws = _ws(c, len(seqs))
    api.check(api.daf_page_free(c.p, len(seqs), _i32(seqs), None if keep is None else _i32(keep), c.t["table"], c.t["refs"], ws))
    assert api.daf_poll_status(ws) == api.DAF_OK
    c.same()


def _compact(c, in_place=True):
    live = _pool(c).compact()
    ws = _ws(c)
    out = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    table, refs = (c.t["table"], c.t["refs"]) if in_place else (torch.full_like(c.t["table"], 99), torch.full_like(c.t["refs"], 99))
    api.check(api.daf_page_compact(c.p, c.t["table"], c.t["refs"], table, refs, out, *c.pool(), ws))
    assert api.daf_poll_status(ws) == api.DAF_OK and out.item() == live
    c.t["table"], c.t["refs"] = table, refs
    # pages that are free now hold what they held or what was moved out of them: only those in use are compared
    used = c.np["refs"] > 0
    for n in ("k8", "v8", "k_scale", "v_scale"):
        assert np.array_equal(c.t[n].cpu().numpy()[:, used], c.np[n][:, used]), n
    c.same(("table", "refs"))
    for n in ("k8", "v8", "k_scale", "v_scale"):
        c.np[n] = c.t[n].cpu().numpy()


@pytest.mark.parametrize("T,Hkv,layers", [(16, 2, 3), (64, 4, 1), (128, 5, 2), (32, 1, 1)])
def test_fork_free_compact_in_turn(T, Hkv, layers):
    c = Cache(60, T, Hkv, 12, 10, n_layers=layers, seed=T, junk=False)
    rng = random.Random(T)
    refused = {"": 0, "bounds": 0, "pages": 0}
    for step in range(60):
        rows = list(range(12))
        empty = [s for s in rows if c.np["table"][s, 0] < 0]
        full = [s for s in rows if s not in empty]
        rng.shuffle(empty)
        what = rng.random()
        if what < 0.5 and empty:
            src, dst, keep, want = [], [], [], []
            for d in empty[:rng.randint(1, 3)]:
                s = rng.choice(full + [-1]) if full else -1
                have = int((c.np["table"][s] >= 0).sum()) * T if s >= 0 else 0
                k = rng.randint(0, have)
                src.append(s); dst.append(d); keep.append(k); want.append(min(10 * T, k + rng.randint(0, 3 * T)))
            refused[_fork(c, src, dst, keep, want, rng.random() < 0.6)] += 1
        elif what < 0.7 and full:
            grow = rng.sample(full, min(len(full), rng.randint(1, 4)))
            keep = [rng.randint(0, int((c.np["table"][s] >= 0).sum()) * T) for s in grow]
            refused[_fork(c, grow, grow, keep, [min(10 * T, k + rng.randint(0, 2 * T)) for k in keep], True)] += 1
        elif what < 0.9 and full:
            some = rng.sample(full, min(len(full), rng.randint(1, 5)))
            _free(c, some, None if rng.random() < 0.5 else [rng.randint(0, 6 * T) for _ in some])
        else:
            _compact(c, in_place=rng.random() < 0.5)
    assert refused[""] > 10


def test_fork_refuses_what_is_not_as_described():
    c = Cache(12, 16, 1, 6, 4, seed=1, junk=False)
    assert _fork(c, [-1, -1], [0, 1], [0, 0], [40, 20], True) == ""
    for src, dst, keep, want in (([-1], [6], [0], [16]), ([-1], [-1], [0], [16]), ([6], [2], [0], [16]), ([0], [2], [-1], [16]),
                                 ([0], [2], [0], [-1]), ([0], [2], [0], [65]), ([0], [2], [65], [64]), ([0], [1], [10], [16]),
                                 ([0], [2], [49], [50]), ([0, 0], [2, 2], [10, 10], [10, 10]), ([0, 2], [2, 3], [10, 10], [10, 10]),
                                 ([0, 0], [0, 2], [40, 40], [64, 40]), ([0], [0], [50], [64]), ([1], [3], [40], [40])):
        assert _fork(c, src, dst, keep, want, True) == "bounds", (src, dst, keep, want)
    assert _fork(c, [-1, -1], [2, 3], [0, 0], [64, 64], True) == "pages"
    assert _fork(c, [-1, -1], [2, 3], [0, 0], [64, 48], True) == ""
    assert _fork(c, [0], [0], [40], [64], True) == "pages"
    _free(c, [2, 2, 3])


def test_large_pool_and_many_items():
    c = Cache(70000, 16, 1, 900, 40, seed=2, junk=False)
    rng = random.Random(5)
    n = 880
    assert _fork(c, [-1] * n, list(range(n)), [0] * n, [rng.randint(0, 640) for _ in range(n)], True) == ""
    _free(c, [s for s in range(n) if rng.random() < 0.6])
    _compact(c)
    full = [s for s in range(n) if c.np["table"][s, 0] >= 0]
    empty = [s for s in range(900) if c.np["table"][s, 0] < 0][:300]
    src = [rng.choice(full) for _ in empty]
    keep = [rng.randint(0, int((c.np["table"][s] >= 0).sum()) * 16) for s in src]
    assert _fork(c, src, empty, keep, [min(640, k + 40) for k in keep], True) == ""
    _compact(c, in_place=False)


@pytest.mark.parametrize("used", [0, 1, 4])
def test_compact_of_an_empty_and_a_full_pool(used):
    c = Cache(4, 16, 2, 2, 4, n_layers=2, seed=3, junk=False)
    if used:
        c.give(1, 16 * used)
    _compact(c)
    _compact(c, in_place=False)


def test_compact_reports_entries_whose_page_has_no_count():
    c = Cache(9, 16, 1, 2, 4, seed=1, junk=False)
    c.np["table"][0, :3] = [8, 6, 7]
    c.np["refs"][[8, 7]] = 1                  # nothing counts page 6
    c.np["table"][1, 0] = 9                   # outside the pool
    c.up()
    ws = _ws(c)
    ws.view(torch.uint8)[256:].fill_(3)       # whatever an earlier call left there
    api.check(api.daf_page_compact(c.p, c.t["table"], c.t["refs"], c.t["table"], c.t["refs"], None, *c.pool(), ws))
    assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
    assert c.t["table"].cpu().tolist() == [[1, -1, 0, -1], [-1, -1, -1, -1]]
    assert c.t["refs"].cpu().tolist() == [1, 1] + [0] * 7


def test_a_table_of_very_many_rows():
    n = 70000
    c = Cache(500, 16, 1, n, 2, seed=2, junk=False)
    assert _fork(c, [-1, -1, -1], [69999, 3, 65536], [0, 0, 0], [32, 17, 5], True) == ""
    assert _fork(c, [69999, 69999, 3], [65537, 0, 69998], [20, 16, 17], [20, 32, 30], True) == ""
    assert _fork(c, [69999, 69999], [65538, 65538], [20, 20], [20, 20], True) == "bounds"
    assert _fork(c, [69999, 65539], [65539, 8], [20, 0], [20, 16], True) == "bounds"
    _free(c, [65536, 69999])
    _compact(c)


def test_free_reports_rows_and_counts_that_are_wrong():
    c = Cache(6, 16, 1, 2, 3, seed=1, junk=False)
    c.give(0, 48)
    c.np["refs"][c.np["table"][0, 1]] = 0
    c.up()
    ws = _ws(c)
    for seqs, keep in (([2], None), ([-1], None), ([0], [-1])):
        api.check(api.daf_page_free(c.p, 1, _i32(seqs), None if keep is None else _i32(keep), c.t["table"], c.t["refs"], ws))
        assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
        c.same()
    api.check(api.daf_page_free(c.p, 1, _i32([0]), None, c.t["table"], c.t["refs"], ws))
    assert api.daf_poll_status(ws) == api.DAF_ERR_BOUNDS
    assert torch.all(c.t["table"] == -1) and torch.all(c.t["refs"] == 0)


# --------------------------------------------------------------------------------------------------------- as they are used
def test_a_context_is_repaired_in_pages_and_answered():
    """Documents in pages -> a copy for this question -> daf_layer over its rows -> repaired and question rows back into the pages ->
    the question's attention over them -> answers forked, decoded token by token in a captured graph, one rolled back -> compact."""
    T, Hkv, Hq, L_d, L_q = 32, 2, 8, 300, 20
    N = L_d + L_q
    c = Cache(64, T, Hkv, 6, 14, seed=31, junk=False)
    c.p.n_layers = 1
    _fork(c, [-1], [0], [0], [L_d], True)
    docs_k, docs_v = _rows(L_d, Hkv, 1, 0.3), _rows(L_d, Hkv, 2, 0.3)
    _write(c, [L_d], [L_d], k=docs_k, v=docs_v)
    _fork(c, [0], [1], [L_d], [N], False)
    # the layer runs on the rows as the pages hold them
    bf = torch.bfloat16
    kv = [torch.zeros(N, Hkv, 128, dtype=bf, device=DEV) for _ in range(2)]
    ws = _ws(c, 4, L_q, Hq)
    api.check(api.daf_page_read(c.p, 0, 1, _i32([1]), None, _i32([0, L_d]), L_d, c.t["table"], *c.pool(), kv[0], kv[1], ws))
    g = torch.Generator().manual_seed(3)
    fresh = [torch.randn(N, h, 128, generator=g).to(bf).to(DEV) for h in (Hq, Hkv, Hkv)]
    lp = api.make_params(L_d, L_q, 0.2, Hq, Hkv)
    k = api.daf_num_important(L_d, 0.2)
    lws = api.alloc_workspace(lp)
    scores = torch.rand(1, L_d, generator=g).to(DEV)
    idx = torch.zeros(k, dtype=torch.int32, device=DEV)
    qp, kp, vp = [torch.zeros(k, h, 128, dtype=bf, device=DEV) for h in (Hq, Hkv, Hkv)]
    hidden = torch.zeros(k + L_q, Hq, 128, dtype=bf, device=DEV)
    api.check(api.daf_layer(lp, scores, 1, None, *fresh, kv[0], kv[1], idx, qp, kp, vp, hidden, None, lws))
    assert api.daf_poll_status(lws) == api.DAF_OK
    where = idx.tolist()
    _write(c, [L_d], [k], idx=where, seqs=[1], k=kp.cpu(), v=vp.cpu())
    _write(c, [N], [L_q], seqs=[1], k=fresh[1][L_d:].cpu(), v=fresh[2][L_d:].cpu())
    c.same()
    got, _ = _attend(c, [N], L_q, Hq, seqs=[1], q=fresh[0][None, L_d:].cpu())
    # ... which is the layer's question stage but for the 8-bit rows: bytes are off by 2^-4 of their values at most
    assert np.linalg.norm(got[0] - hidden[k:].float().cpu().numpy()) <= 0.1 * np.linalg.norm(got[0])
    # three answers, four tokens each, one graph replayed
    ans = [2, 3, 4]
    _fork(c, [1] * 3, ans, [N] * 3, [N + 8] * 3, True)
    lens, row_off, seqs = _i32([N] * 3), _i32([0, 1, 2, 3]), _i32(ans)
    q = torch.zeros(3, 1, Hq, 128, dtype=bf, device=DEV)
    nk, nv, out = torch.zeros(3, Hkv, 128, dtype=bf, device=DEV), torch.zeros(3, Hkv, 128, dtype=bf, device=DEV), torch.zeros(3, 1, Hq, 128, dtype=bf, device=DEV)

    def step():
        lens.add_(1)
        api.check(api.daf_page_write(c.p, 0, 3, seqs, lens, row_off, None, 1, nk, nv, c.t["table"], c.t["refs"], *c.pool(), ws))
        api.check(api.daf_page_attn(c.p, 0, 3, seqs, lens, 1, Hq, 0.0, q, c.t["table"], *c.pool(), out, None, ws))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    saved = {n: t.clone() for n, t in c.t.items()}
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    for n, t in c.t.items():
        t.copy_(saved[n])
    lens.fill_(N)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lens.fill_(N)
    for i in range(4):
        x = [torch.randn(t.shape, generator=g).to(bf) for t in (q, nk, nv)]
        for t, y in zip((q, nk, nv), x):
            t.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for n, rows in (("k", x[1]), ("v", x[2])):
            O.write(c.np[n + "8"], c.np[n + "_scale"], 0, ans, [N + i + 1] * 3, [0, 1, 2, 3], None, rows.float().numpy(), c.np["table"])
        c.same()
        again, _ = _attend(c, [N + i + 1] * 3, 1, Hq, seqs=ans, q=x[0])
        assert np.array_equal(again, out.float().cpu().numpy())
    assert api.daf_poll_status(ws) == api.DAF_OK
    _free(c, [3, 4], [0, N + 1])              # an answer ends, another loses its last three tokens
    _free(c, [0])
    _compact(c)
    _fork(c, [4], [4], [N + 1], [N + 40], True)
    _attend(c, [N, N + 4, N + 1], 1, Hq, seqs=[1, 2, 4])


def test_calls_on_another_stream_and_two_at_once():
    lens = [900, 40, 333]
    c = _cache_for(lens, 64, 4, seed=41, junk=False)
    base = {L_q: _attend(c, lens, L_q, 28, check=False)[0] for L_q in (1, 25)}
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    qs = {L_q: torch.randn(3, L_q, 28, 128, generator=torch.Generator().manual_seed(100)).to(torch.bfloat16).to(DEV) for L_q in (1, 25)}
    outs = [torch.zeros(3, L_q, 28, 128, dtype=torch.bfloat16, device=DEV) for L_q in (1, 25)]
    wss = [_ws(c, 3, L_q, 28) for L_q in (1, 25)]
    l = _i32(lens)
    torch.cuda.synchronize()
    for _ in range(20):
        for i, L_q in enumerate((1, 25)):
            api.check(api.daf_page_attn(c.p, 0, 3, None, l, L_q, 28, 0.0, qs[L_q], c.t["table"], *c.pool(), outs[i], None, wss[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i, L_q in enumerate((1, 25)):
        assert api.daf_poll_status(wss[i]) == api.DAF_OK
        assert np.array_equal(outs[i].float().cpu().numpy(), base[L_q])


def test_two_graphs_share_a_workspace():
    c = _cache_for([700, 90], 16, 2, seed=51, junk=False)
    ws = _ws(c, 2, 30, 8)
    lens = _i32([700, 90])
    q = {L_q: torch.randn(2, L_q, 8, 128, generator=torch.Generator().manual_seed(100)).to(torch.bfloat16).to(DEV) for L_q in (1, 30)}
    out = {L_q: torch.zeros(2, L_q, 8, 128, dtype=torch.bfloat16, device=DEV) for L_q in (1, 30)}
    graphs = {}
    for L_q in (1, 30):
        api.check(api.daf_page_attn(c.p, 0, 2, None, lens, L_q, 8, 0.0, q[L_q], c.t["table"], *c.pool(), out[L_q], None, ws))
        torch.cuda.synchronize()
        graphs[L_q] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[L_q]):
            api.check(api.daf_page_attn(c.p, 0, 2, None, lens, L_q, 8, 0.0, q[L_q], c.t["table"], *c.pool(), out[L_q], None, ws))
    for now in ([700, 90], [13, 64], [0, 1], [700, 90]):
        lens.copy_(_i32(now))
        for L_q in (1, 30):
            out[L_q].fill_(7.0)
            graphs[L_q].replay()
        torch.cuda.synchronize()
        for L_q in (1, 30):
            got, _ = _attend(c, now, L_q, 8)
            assert np.array_equal(got, out[L_q].float().cpu().numpy())
    assert api.daf_poll_status(ws) == api.DAF_OK


@pytest.mark.parametrize("L_q", [1, 6, 7, 40, 80])          # rows of a KV head: 4, 24 | 28, 160, 320 (one tile, a pair, a pair and one)
@pytest.mark.parametrize("exps", [(-60, -59), (-60, -3), (-14, -9)])
def test_zero_and_tiny_rows_over_small_key_scales(L_q, exps):
    lens = [500, 3, 0, 200]                                 # (3 and 0: rows that see nothing)
    c = _cache_for(lens, 16, 2, seed=61, junk=False)
    c.np["k_scale"][:] = (2.0 ** np.random.default_rng(L_q).integers(*exps, c.np["k_scale"].shape)).astype(np.float32)
    c.up()
    q = torch.randn(4, L_q, 8, 128, generator=torch.Generator().manual_seed(5))
    q[:, :, ::4] = 0.0
    q[:, :, 1::4] *= 1e-30
    q[:, :, 2::4] *= 1e-37
    q[3, -1] = 0.0
    for scale in (0.0, 1e-6):
        _attend(c, lens, L_q, 8, q=q.to(torch.bfloat16), scale=scale)


@pytest.mark.parametrize("L_q", [1, 7, 70])
def test_zero_keys_as_they_are_written(L_q):
    lens = [150, 5, 64]
    c = _cache_for(lens, 32, 1, seed=62, junk=False)
    k = _rows(sum(lens), 1, 3)
    k[40:150] = 0.0
    k[155:] = 0.0
    _write(c, lens, lens, k=k)
    c.same()
    assert (c.np["k_scale"] == 2.0 ** -60).any()
    q = torch.randn(3, L_q, 4, 128, generator=torch.Generator().manual_seed(6))
    q[:, :, 1] = 0.0
    q[:, :, 2] *= 1e-25
    _attend(c, lens, L_q, 4, q=q.to(torch.bfloat16))


@pytest.mark.parametrize("T", [16, 128])
@pytest.mark.parametrize("with_refs", [True, False])
def test_growth_replaces_the_page_of_the_next_token_at_a_border_too(T, with_refs):
    c = Cache(8, T, 2, 3, 4, n_layers=2, seed=T, junk=False)
    assert _fork(c, [-1], [0], [0], [2 * T], True) == ""
    _write(c, [2 * T], [2 * T], layer=1)
    assert _fork(c, [0], [1], [2 * T], [2 * T], True) == ""
    assert c.t["table"].tolist() == [[0, 1, -1, -1], [0, 1, -1, -1], [-1] * 4] and c.t["refs"].tolist()[:3] == [2, 2, 0]
    # row 0 loses its second page's tokens by its length alone; its next token must not go into what row 1 still has
    assert _fork(c, [0], [0], [T], [2 * T], True) == ""
    assert c.t["table"].tolist() == [[0, 2, -1, -1], [0, 1, -1, -1], [-1] * 4] and c.t["refs"].tolist()[:4] == [2, 1, 1, 0]
    child = {n: c.t[n][:, 1].clone() for n in ("k8", "v8", "k_scale", "v_scale")}
    _write(c, [T + 1], [1], layer=1, refs=with_refs)
    c.same()
    assert all(torch.equal(c.t[n][:, 1], x) for n, x in child.items())


def test_growth_of_rows_set_back_further():
    T = 16
    c = Cache(12, T, 1, 6, 6, seed=4, junk=False)
    assert _fork(c, [-1], [0], [0], [5 * T], True) == ""
    assert _fork(c, [0, 0, 0], [1, 2, 3], [5 * T] * 3, [5 * T] * 3, True) == ""
    # several rows at once: at a border, inside a page, at the begin, at the end of what the row holds
    assert _fork(c, [0, 1, 2, 3], [0, 1, 2, 3], [2 * T, 2 * T + 5, 0, 5 * T], [2 * T + 1, 6 * T, 1, 6 * T], True) == ""
    assert c.t["table"][:4].tolist() == [[0, 1, 5, 3, 4, -1], [0, 1, 6, 3, 4, 7], [8, 1, 2, 3, 4, -1], [0, 1, 2, 3, 4, 9]]
    assert c.t["refs"].tolist() == [3, 4, 2, 4, 4, 1, 1, 1, 1, 1, 0, 0]
    # pages of one's own stay; the length may stay as well
    assert _fork(c, [0, 2], [0, 2], [2 * T, 5], [2 * T, 5], True) == ""
    assert c.t["table"][:3:2].tolist() == [[0, 1, 5, 3, 4, -1], [8, 1, 2, 3, 4, -1]]
    # both owners of a page at once: each gets one
    _free(c, [1, 2])
    assert _fork(c, [0, 3], [0, 3], [3 * T, 3 * T], [3 * T + 1] * 2, True) == ""
    assert _fork(c, [-1], [4], [0], [4 * T], True) == ""
    # a page more is needed than there is: nothing changes
    assert _fork(c, [0], [0], [T], [5 * T], True) == "pages"


@pytest.mark.parametrize("share", [True, False])
@pytest.mark.parametrize("hole", [-1, -7, 40, 10 ** 9])
def test_a_source_row_with_a_hole_changes_nothing(hole, share):
    c = Cache(40, 16, 2, 8, 12, n_layers=2, seed=6, junk=False)
    for s in (0, 1):
        c.give(s, 150, up=False)
    c.np["table"][0, 4] = hole
    c.up()
    for src, dst, keep, want in (([0], [2], [150], [160]), ([0], [2], [80], [80]), ([0], [2], [65], [65]), ([1, 0, 1], [2, 3, 4], [20, 130, 3], [40, 130, 3])):
        assert _fork(c, src, dst, keep, want, share) == "bounds", (src, keep)
    # what lies behind the kept tokens does not count
    assert _fork(c, [0, 1], [2, 3], [64, 150], [70, 160], share) == ""
    # a row that grows: the page its next token goes into counts
    if hole > 0:
        assert _fork(c, [0], [0], [66], [70], True) == "bounds"
        assert _fork(c, [0], [0], [64], [70], True) == "bounds"


@pytest.mark.parametrize("at", [0, 31, 255, 256, 300, 698])
def test_a_hole_anywhere_in_long_rows_of_many_items(at):
    c = Cache(1500, 16, 1, 60, 700, seed=7, junk=False)
    c.give(0, 699 * 16, up=False)
    c.give(1, 699 * 16, up=False)
    c.np["table"][1, at] = -1 if at < 300 else 1500
    c.up()
    n = 50
    assert _fork(c, [0] * (n - 1) + [1], list(range(2, n + 2)), [699 * 16] * n, [699 * 16] * n, True) == "bounds"
    assert _fork(c, [0] * n, list(range(2, n + 2)), [699 * 16] * n, [699 * 16 + 1] * n, True) == ""


def test_a_hole_that_only_some_of_a_rows_items_keep():
    c = Cache(60, 16, 1, 12, 10, seed=8, junk=False)
    c.give(0, 150, up=False)
    c.np["table"][0, 7] = -1
    c.up()
    for keep in ([60, 40, 130, 20], [130, 20, 20, 20], [20, 20, 20, 113], [20, 130, 140, 150]):
        assert _fork(c, [0] * 4, [2, 3, 4, 5], keep, keep, True) == "bounds", keep
    # an item before that keeps more, but is none of a row's sources, covers nothing
    assert _fork(c, [-1, 0], [2, 3], [150, 120], [10, 120], True) == "bounds"
    assert _fork(c, [0] * 4, [2, 3, 4, 5], [112, 40, 112, 20], [112, 112, 112, 112], True) == ""


def test_host_memory_is_refused_unless_it_is_pinned():
    lens = [100, 40]
    c = _cache_for(lens, 16, 2, seed=64, junk=False)
    want, _ = _attend(c, lens, 1, 4, check=False)
    q = torch.randn(2, 1, 4, 128, generator=torch.Generator().manual_seed(100)).to(torch.bfloat16).to(DEV)
    out, ws = torch.zeros_like(q), _ws(c, 2, 1, 4)
    host = torch.tensor(lens, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        api.daf_page_attn(c.p, 0, 2, None, host, 1, 4, 0.0, q, c.t["table"], *c.pool(), out, None, ws)
    with pytest.raises(ValueError, match="int64"):
        api.daf_page_attn(c.p, 0, 2, None, _i32(lens).long(), 1, 4, 0.0, q, c.t["table"], *c.pool(), out, None, ws)
    api.check(api.daf_page_attn(c.p, 0, 2, None, host.pin_memory(), 1, 4, 0.0, q, c.t["table"], *c.pool(), out, None, ws))
    assert api.daf_poll_status(ws) == api.DAF_OK and np.array_equal(out.float().cpu().numpy(), want)


@pytest.mark.parametrize("L_q", [1, 6, 7, 70])
@pytest.mark.parametrize("q_scale", [1.0, 25.0])
def test_value_scales_at_the_ends_of_their_range(L_q, q_scale):
    lens = [700, 129, 2000]
    c = _cache_for(lens, 16, 2, seed=63, junk=False)
    ends = np.array([2.0 ** -60, 2.0 ** 30], np.float32)
    c.np["v_scale"][:] = ends[np.random.default_rng(1).integers(0, 2, c.np["v_scale"].shape)]
    c.up()
    _attend(c, lens, L_q, 8, q_scale=q_scale)
    for end in ends:                                       # ... and all alike
        c.np["v_scale"][:] = end
        c.up()
        _attend(c, lens, L_q, 8, q_scale=q_scale)


@pytest.mark.parametrize("L_q", [1, 6, 7, 70])
@pytest.mark.parametrize("bad", [2.0 ** -61, 2.0 ** 31, 1.01 * 2.0 ** 30, 0.0, -2.0, math.inf, math.nan])
def test_value_scales_outside_their_range_are_reported(L_q, bad):
    lens = [200, 90, 33]
    c = _cache_for(lens, 16, 2, seed=65, junk=False)
    good = c.np["v_scale"].copy()
    for seq, page, head in ((0, 0, 0), (0, 12, 1), (1, 3, 0), (2, 2, 1)):
        c.np["v_scale"][:] = good
        c.np["v_scale"][0, c.np["table"][seq, page], head] = bad
        c.up()
        _attend(c, lens, L_q, 8, status=api.DAF_ERR_BOUNDS, check=False)
        # where nobody sees the page it does not count
        shorter = [min(L, 16 * page) if b == seq else L for b, L in enumerate(lens)]
        _attend(c, shorter, L_q, 8, check=False)


@pytest.mark.parametrize("n,L_q,Hq,Hkv,T,lo,hi", [(10, 15, 40, 8, 32, 964, 10986), (16, 7, 40, 8, 32, 2049, 3689), (12, 64, 16, 2, 16, 300, 6000),
                                                  (40, 30, 8, 4, 128, 0, 700), (3, 130, 28, 4, 64, 500, 9000)])
def test_many_launches_give_the_same_bits(n, L_q, Hq, Hkv, T, lo, hi):
    """Pieces of work in whatever order their bytes arrive: after a write to the workspace, after other data in L2, back to back."""
    rng = random.Random(n)
    c = _cache_for([rng.randint(lo, hi) for _ in range(n)], T, Hkv, seed=66, junk=False)
    lens = _i32([int((c.np["table"][s] >= 0).sum()) * T - rng.randint(0, T - 1) if c.np["table"][s, 0] >= 0 else 0 for s in range(n)])
    q = torch.randn(n, L_q, Hq, 128, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).to(DEV)
    ws, other = _ws(c, n, L_q, Hq), torch.empty(64 << 20, device=DEV)
    first = None
    for i in range(120):
        if i % 3 == 1:
            ws[256:].random_(0, 255)
        if i % 3 == 2 and i < 60:
            other.fill_(i)
        out, lse = torch.full_like(q, 7.0), torch.full((n, Hq, L_q), 7.0, device=DEV)
        api.check(api.daf_page_attn(c.p, 0, n, None, lens, L_q, Hq, 0.0, q, c.t["table"], *c.pool(), out, lse, ws))
        if first is None:
            first = out, lse
            continue
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), (i, (out != first[0]).any(-1).nonzero()[:3].tolist())
    assert api.daf_poll_status(ws) == api.DAF_OK


@pytest.mark.parametrize("L_q,Hq", [(1, 2), (3, 8), (1, 24), (13, 2), (25, 8)])
@pytest.mark.parametrize("n", [1, 40])
def test_nan_in_a_part_that_hardly_counts(L_q, Hq, n):
    """Logits hundreds apart: parts of a row that several warps or CTAs worked on get a weight of 0, and a NaN in one has to stay."""
    lens = [3000] if n == 1 else [100 + 13 * i for i in range(n)]
    c = _cache_for(lens, 16, 1, seed=67, junk=False)
    rng = np.random.default_rng(3)
    for seq, L in enumerate(lens):
        for j in rng.integers(0, max(1, L - L_q), 2 if n == 1 else 1):
            x = "k8" if (seq + n) % 3 == 0 else "v8"
            c.np[x][0, c.np["table"][seq, j // 16], 0, j % 16, rng.integers(0, 128)] = 0x7F
    c.up()
    _attend(c, lens, L_q, Hq, scale=0.3, q_scale=3.0)
    c.np["k8"][0, c.np["table"][0, 5], 0, 3, 1] = 0xFF
    c.up()
    _attend(c, lens, L_q, Hq, scale=0.3, q_scale=3.0, seed=1)


@pytest.mark.parametrize("T,L,L_q,Hq,page", [(16, 1000, 200, 8, 61), (32, 3, 53, 25, 0), (64, 500, 64, 16, 7), (16, 300, 299, 4, 18)])
def test_a_missing_page_that_only_later_rows_see_is_reported(T, L, L_q, Hq, page):
    c = _cache_for([L, 40], T, 1, seed=68, junk=False)
    for gone in (-1, c.n_pages):
        c.np["table"][0, page] = gone
        c.up()
        _attend(c, [L, 40], L_q, Hq, status=api.DAF_ERR_BOUNDS)


@pytest.mark.parametrize("T", [16, 128])
def test_read_of_scales_at_the_ends_of_the_range(T):
    """Products below 2^-126 among them: rounded to bf16's subnormal numbers, as daf_expand_fp8_cache does."""
    n = 2560 // T
    c = Cache(n, T, 1, 1, n, seed=T, junk=False)
    c.np["k8"][:] = (np.arange(n * T * 128) * 37 % 256).astype(np.uint8).reshape(c.np["k8"].shape)
    c.np["v8"][:] = c.np["k8"][:, ::-1]
    for x, lo in (("k", -126), ("v", -121)):
        c.np[x + "_scale"][:] = (2.0 ** (lo + np.arange(n) % 9)).astype(np.float32).reshape(c.np[x + "_scale"].shape)
    c.np["v_scale"][0, ::4] *= np.float32(1.37)
    c.np["k_scale"][0, 5] = 2.0 ** 119
    c.give(0, n * T)
    k = torch.zeros(n * T, 1, 128, dtype=torch.bfloat16, device=DEV)
    v, ws = torch.zeros_like(k), _ws(c)
    api.check(api.daf_page_read(c.p, 0, 1, None, None, _i32([0, n * T]), n * T, c.t["table"], *c.pool(), k, v, ws))
    assert api.daf_poll_status(ws) == api.DAF_OK
    for x, got in (("k", k), ("v", v)):
        want = O.read(c.np[x + "8"], c.np[x + "_scale"], 0, 0, 0, n * T, c.np["table"])
        assert np.array_equal(got.float().cpu().numpy(), want, equal_nan=True), x
        assert ((want != 0) & (np.abs(want) < 2.0 ** -126)).any()


@pytest.mark.parametrize("L_q", [1, 6, 7, 70])
@pytest.mark.parametrize("k_exp,q_exp", [(-126, 0), (-126, 100), (90, -92), (119, -121), (-60, 60)])
def test_key_scales_at_the_ends_of_their_range(L_q, k_exp, q_exp):
    lens = [700, 4, 90]
    c = _cache_for(lens, 32, 2, seed=69, junk=False)
    c.np["k_scale"][:] = 2.0 ** k_exp
    c.np["k_scale"][0, ::3] *= np.float32(1.37)
    c.up()
    _attend(c, lens, L_q, 8, q_scale=2.0 ** q_exp)
