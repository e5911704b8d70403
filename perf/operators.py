"""The operators of the paged 8-bit cache as timed cases, with their plain forms.

A program that serves answers over repaired contexts keeps the K/V rows of all its sequences in pages of 16 to 128 tokens, one
byte per element (1 sign, 4 exponent, 3 mantissa bits) and one fp32 scale per page and KV head:

  k8, v8            [layers, pages, KV heads, tokens of a page, 128] bytes,    k_scale, v_scale  [layers, pages, KV heads]
  table             int32 [sequences, max_pages] page numbers, -1 behind a sequence's last page
  refs              int32 [pages] how many table entries name a page (0: free)

Kinds of pass (`case["kind"]`):
  write     bf16 rows put into the pages of one layer: the newest tokens of every sequence, or rows at given positions
  read      a sequence's tokens as bf16 rows, as daf_layer takes a cache
  attn      the newest L_q tokens of every sequence attend its pages (one token: a decoding step; many: a further question)
  fork      answers that have ended give their pages back, new ones start from their context's pages
  compact   the pages in use move to the front of the pool
Heads, contexts and questions are those of the repository's own workloads (28/4, 32/8 and 40/8 heads of 128 channels, 1k to 32k
tokens of context, questions of some tens of tokens).
"""
import math

import torch

own = False

D = 128
HEADS = {"28/4": (28, 4), "32/8": (32, 8), "40/8": (40, 8)}
E4M3 = torch.float8_e4m3fn
MIN_SCALE = 2.0 ** -60
WORKSPACE = 64 << 20      # more than daf_page_workspace_bytes of every case below


def _case(kind, heads, T, n, lo, hi, **kw):
    c = {"kind": kind, "heads": heads, "T": T, "n": n, "lo": lo, "hi": hi, "layers": 1, "rows": 0, "every": 0, "L_q": 1,
         "share": True, "ask": 0}
    return dict(c, **kw)


def listed():
    def named(name, *a, **kw):
        return dict(_case(*a, **kw), name=name)

    return [
        # one decoding step of 64 answers: a row each, most into a page that is in use
        named("write_token_64_sequences", "write", "32/8", 16, 64, 500, 12000, rows=1),
        # a layer's share of a context that has just been computed, into its pages
        named("write_context_16k", "write", "32/8", 64, 1, 16384, 16384, rows=16384),
        # a short context on its way into daf_layer, and the longest of the benchmark's
        named("read_6k", "read", "28/4", 64, 1, 6208, 6208),
        named("read_32k_ragged", "read", "28/4", 128, 1, 32811, 32811),
        # the first tokens of one answer over a short context: latency
        named("decode_1_over_1k", "attn", "28/4", 64, 1, 1057, 1057),
        # one answer over the benchmark's longest document set
        named("decode_1_over_32k", "attn", "28/4", 64, 1, 32899, 32899),
        # a batch of answers of all lengths, small pages
        named("decode_64_ragged", "attn", "32/8", 16, 64, 500, 12000),
        # a further question over a 32k context: tensor-core time
        named("question_128_over_32k", "attn", "28/4", 64, 1, 32896, 32896, L_q=128),
        # eight answers to one question start from its context, every layer: pages shared, the last one copied
        named("fork_8_answers", "fork", "28/4", 64, 8, 6208, 6227, layers=28, ask=256),
        # copies of four contexts whose rows are going to be repaired in place
        named("copy_4_contexts", "fork", "32/8", 64, 4, 4000, 4200, layers=8, share=False, ask=128),
        # a small pool with some holes; a large one of which half of the sequences have gone
        named("compact_small", "compact", "28/4", 16, 12, 300, 1500, layers=2),
        named("compact_large", "compact", "32/8", 64, 24, 2000, 8000, layers=4),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads, T = rng.choice(sorted(HEADS)), rng.choice((16, 32, 64, 128))
    kind = rng.choice(("write", "write", "read", "attn", "attn", "attn", "fork", "compact"))
    if kind == "write":
        how = rng.choice(("token", "context", "given"))
        if how == "token":
            n = log(1, 64)
            return _case(kind, heads, T, n, log(20, 1000), log(1001, 12000), rows=log(1, 20))
        L = log(200, 14000)
        return _case(kind, heads, T, 1, L, L, rows=L) if how == "context" else _case(kind, heads, T, 1, L, L, every=rng.randint(2, 19))
    if kind == "read":
        L = log(100, 32000)
        return _case(kind, heads, T, 1, L, L)
    if kind == "attn":
        how = rng.choice(("token", "few", "question"))
        if how == "token":
            n = log(1, 64)
            top = log(200, min(60000, 700000 // n))
            return _case(kind, heads, T, n, min(top, log(1, 5000)), top)
        if how == "few":
            n = log(1, 32)
            top = log(200, min(30000, 300000 // n))
            return _case(kind, heads, T, n, min(top, log(50, 5000)), top, L_q=rng.randint(2, 16))
        L = log(500, 20000)
        return _case(kind, heads, T, 1, L, L, L_q=min(L, log(17, 150)))
    if kind == "fork":
        lo = log(100, 3000)
        return _case(kind, heads, T, rng.randint(1, 8), lo, lo + log(1, 1200), layers=rng.randint(1, 8), share=rng.random() < 0.5, ask=log(1, 600))
    lo = log(50, 2000)
    return _case(kind, heads, T, rng.randint(2, 24), lo, lo + log(1, 6000), layers=rng.randint(1, 4))


def _lens(case):
    """The sequences' lengths: spread over lo .. hi in no order."""
    lo, hi = case["lo"], case["hi"]
    lens = [lo + int((hi - lo) * ((0.35 + i * 0.6180339887498949) % 1.0)) for i in range(case["n"])]
    return lens if len(lens) > 1 else [hi]


def _counts(case):
    """Rows written to each sequence."""
    return [min(case["rows"], L) if not case["every"] else len(range(case["every"] // 2, L, case["every"])) for L in _lens(case)]


def _pages(tokens, T):
    return -(-tokens // T)


def work(case):
    Hq, Hkv = HEADS[case["heads"]]
    T, lens, layers = case["T"], _lens(case), case["layers"]
    page = 2 * layers * Hkv * (T * D + 4)            # K and V of one page in all layers, with their scales
    if case["kind"] == "write":
        rows = sum(_counts(case))
        return {"bytes": rows * Hkv * D * 2 * 3, "flops": rows * Hkv * D * 2}
    if case["kind"] == "read":
        return {"bytes": sum(lens) * Hkv * D * 2 * 3, "flops": sum(lens) * Hkv * D * 2}
    if case["kind"] == "attn":
        L_q = case["L_q"]
        keys = sum(max(0, L - L_q + t + 1) for L in lens for t in range(L_q))
        return {"bytes": 2 * Hkv * D * sum(lens) + case["n"] * L_q * Hq * (4 * D + 4), "flops": 4 * D * Hq * keys}
    if case["kind"] == "fork":
        new = [_pages(L + case["ask"], T) for L in lens]
        copied = [_pages(L, T) - (L // T if case["share"] else 0) for L in lens]
        return {"bytes": sum(copied) * 2 * page + 4 * 2 * sum(new), "flops": 0}
    pool, held, moved = _fragments(case)
    return {"bytes": moved * 2 * page + 2 * 4 * (pool + sum(held)), "flops": 0}


def _fragments(case):
    """Pages of a pool whose sequences came and went: (pages in all, pages of each sequence that stays, pages that have to move)."""
    held, at = [], 0
    used = []
    for i, L in enumerate(_lens(case)):
        n = _pages(L, case["T"])
        if i % 2:                                     # every other sequence has gone
            held.append(n)
            used += range(at, at + n)
        at += n
    live = sum(held)
    return at, held, sum(p >= live for p in used)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    Hq, Hkv = HEADS[case["heads"]]
    T, lens, layers, n = case["T"], _lens(case), case["layers"], case["n"]
    kind = case["kind"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    ints = dict(dtype=torch.int32, device=dev)
    s = {"kind": kind, "heads": (Hq, Hkv), "T": T, "layers": layers, "n": n, "max_len": max(lens), "case": dict(case)}
    if kind == "compact":
        n_pages, held, _ = _fragments(case)
        max_pages = max(held)
        table = torch.full((len(held), max_pages), -1, **ints)
        refs = torch.zeros(n_pages, **ints)
        at, row = 0, 0
        for i, L in enumerate(lens):
            m = _pages(L, T)
            if i % 2:
                table[row, :m] = torch.arange(at, at + m, **ints).flip(0) if row % 3 == 1 else torch.arange(at, at + m, **ints)
                refs[at:at + m] = 1
                row += 1
            at += m
        s["table_out"], s["refs_out"], s["live"] = torch.empty_like(table), torch.empty_like(refs), torch.zeros(1, **ints)
        s["n_seqs"] = len(held)
    else:
        # each sequence's pages lie where the allocator found them: in no order
        per = [_pages(L, T) for L in lens]
        max_pages = max(per) + (_pages(case["ask"], T) if kind == "fork" else 0) + 1
        rows = 2 * n if kind == "fork" else n
        spare = sum(_pages(L + case["ask"], T) for L in lens) + 3 if kind == "fork" else 3
        n_pages = sum(per) + spare
        order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
        table = torch.full((rows, max_pages), -1, **ints)
        refs = torch.zeros(n_pages, **ints)
        at = 0
        for b, m in enumerate(per):
            table[b, :m] = order[at:at + m]
            at += m
        refs[order[:at].long()] = 1
        s["n_seqs"] = rows
    s.update(n_pages=n_pages, max_pages=max_pages, table=table, refs=refs)
    # a pool as earlier writes left it: values that fill the 8-bit range, scales by how large a page's rows were; K has a few
    # channels larger than the others
    shape = (layers, n_pages, Hkv, T, D)
    for x in "kv":
        pool = torch.empty(shape, dtype=torch.uint8, device=dev)
        for l in range(layers):
            for p0 in range(0, n_pages, 4096):
                part = pool[l, p0:p0 + 4096]
                v = normal(*part.shape) * 64.0
                if x == "k":
                    v[..., 5::32] *= 2.0
                part.copy_(v.clamp_(-448, 448).to(E4M3).view(torch.uint8))
        s[x + "8"] = pool
        s[x + "_scale"] = torch.exp2(torch.randint(-7, -5, shape[:3], generator=gen, device=dev).float())
    s["lens"] = torch.tensor(lens, **ints)
    s["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device=dev)
    bf = torch.bfloat16
    if kind == "write":
        counts = _counts(case)
        s["row_off"] = torch.tensor([0] + counts, **ints).cumsum(0).to(torch.int32)
        s["max_rows"] = max(counts)
        R = sum(counts)
        # rows of unequal size: now and then one that its page's scale does not hold
        s["k"] = (normal(R, Hkv, D) * torch.exp(0.7 * normal(R, 1, 1))).to(bf)
        s["v"] = (normal(R, Hkv, D) * torch.exp(0.7 * normal(R, 1, 1))).to(bf)
        s["idx"] = None
        if case["every"]:
            s["idx"] = torch.arange(case["every"] // 2, lens[0], case["every"], **ints)
    if kind == "read":
        s["row_off"] = torch.tensor([0] + lens, **ints).cumsum(0).to(torch.int32)
        s["max_rows"] = max(lens)
        s["k_rows"] = torch.empty(sum(lens), Hkv, D, dtype=bf, device=dev)
        s["v_rows"] = torch.empty_like(s["k_rows"])
    if kind == "attn":
        s["q"] = normal(n, case["L_q"], Hq, D).to(bf)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(n, Hq, case["L_q"], device=dev)
    if kind == "fork":
        s["src"], s["dst"] = torch.arange(n, **ints), torch.arange(n, 2 * n, **ints)
        s["keep"] = torch.tensor(lens, **ints)
        s["want"] = s["keep"] + case["ask"]
        s["share"] = case["share"]
    return s


# ------------------------------------------------------------------------------------------------------------- plain forms
def _pow2_scale(amax):
    """The least power of two that brings amax into the 8-bit range (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(amax)
    return torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875).int()).clamp_min(MIN_SCALE)


def _plain_write(s):
    T, n_pages, Hkv = s["T"], s["n_pages"], s["heads"][1]
    dev = s["k"].device
    R = s["k"].shape[0]
    off = s["row_off"].long()
    r = torch.arange(R, device=dev)
    b = torch.searchsorted(off, r, right=True) - 1
    lens = s["lens"].long()
    kept_to = lens if s["idx"] is not None else lens - (off[1:] - off[:-1])
    pos = s["idx"].long() if s["idx"] is not None else kept_to[b] + r - off[b]
    slot = pos % T
    page = s["table"].long()[b, pos // T]
    first = torch.zeros(n_pages, dtype=torch.long, device=dev).index_put_((page,), pos - slot)
    limit = torch.zeros(n_pages, dtype=torch.long, device=dev).index_put_((page,), kept_to[b])
    written = torch.zeros(n_pages, T, dtype=torch.bool, device=dev)
    written[page, slot] = True
    kept = (first[:, None] + torch.arange(T, device=dev) < limit[:, None]) & ~written
    touched = written.any(1)[:, None]
    keeps = kept.any(1)[:, None]
    for x in "kv":
        rows = s[x].float()
        size = rows.abs().amax(-1)                                              # [R, Hkv]
        amax = torch.zeros(n_pages, Hkv, device=dev).index_reduce_(0, page, size, "amax")
        old = s[x + "_scale"][0]
        need = _pow2_scale(amax)
        new = torch.where(touched, torch.where(keeps, torch.maximum(need, old), need), old)
        pool = s[x + "8"][0]
        again = (pool.view(E4M3).float() * (old / new)[..., None, None]).to(E4M3).view(torch.uint8)
        pool.copy_(torch.where(kept[:, None, :, None] & touched[..., None, None], again, pool))
        pool[page, :, slot] = (rows / new[page][..., None]).to(E4M3).view(torch.uint8)
        old.copy_(new)
    return _pool(s)


def _pool(s):
    return s["k8"].view(E4M3), s["v8"].view(E4M3), s["k_scale"], s["v_scale"]


def _plain_read(s):
    T = s["T"]
    page = s["table"][0, :_pages(s["max_len"], T)].long()
    for x in "kv":
        wide = s[x + "8"][0][page].view(E4M3).float() * s[x + "_scale"][0][page][..., None, None]
        s[x + "_rows"].copy_(wide.transpose(1, 2).reshape(-1, s["heads"][1], D)[:s["max_len"]])
    return s["k_rows"], s["v_rows"]


def _plain_attn(s):
    (Hq, Hkv), T, n = s["heads"], s["T"], s["n"]
    L_q = s["q"].shape[1]
    page = s["table"][:, :_pages(s["max_len"], T)].long().clamp_min(0)
    wide = []
    at = torch.arange(page.shape[1] * T, device=page.device)
    there = at < s["lens"][:, None]                                             # [n, L]
    for x in "kv":
        w = s[x + "8"][0][page].view(E4M3).float() * s[x + "_scale"][0][page][..., None, None]
        w = w.transpose(1, 2).reshape(n, Hkv, -1, D)
        wide.append(w.masked_fill_(~there[:, None, :, None], 0.0))
    q = s["q"].float().view(n, L_q, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, -1, D)
    z = (q @ wide[0].transpose(-1, -2)) / math.sqrt(D)
    last = s["lens"][:, None].long() - L_q + torch.arange(L_q, device=page.device)   # [n, L_q] last key a row sees
    hidden = (at > last[..., None]).repeat(1, Hq // Hkv, 1)[:, None]            # rows are (head of the group, token)
    z = z.masked_fill_(hidden, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = (p @ wide[1]) / torch.where(total == 0, 1.0, total)
    s["out"].copy_(o.view(n, Hkv, Hq // Hkv, L_q, D).permute(0, 3, 1, 2, 4).reshape(n, L_q, Hq, D))
    s["lse"].copy_((top + torch.log(total)).view(n, Hq, L_q))
    return s["out"], s["lse"]


def _plain_fork(s):
    T, table, refs = s["T"], s["table"], s["refs"]
    src, dst = s["src"].long(), s["dst"].long()
    gone = table[dst]
    refs.index_add_(0, gone[gone >= 0].long(), -torch.ones_like(gone[gone >= 0]))
    col = torch.arange(s["max_pages"], device=table.device)
    keep, want = s["keep"].long()[:, None], s["want"].long()[:, None]
    shared = (col < keep // T) if s["share"] else torch.zeros_like(col, dtype=torch.bool).expand(len(src), -1)
    new = (col < -(-want // T)) & ~shared
    free = torch.nonzero(refs == 0).view(-1)
    fresh = free[(new.view(-1).cumsum(0) - 1).clamp_min(0)].view(new.shape)
    from_ = table[src].long()
    table[dst] = torch.where(shared, from_, torch.where(new, fresh, -1)).to(torch.int32)
    refs.index_add_(0, from_[shared], torch.ones_like(from_[shared], dtype=torch.int32))
    refs[fresh[new]] = 1
    copied = new & (col < -(-keep // T))
    for x in ("k8", "v8", "k_scale", "v_scale"):
        s[x][:, fresh[copied]] = s[x][:, from_[copied]]
    return (table, refs) + _pool(s)


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    used = refs > 0
    live = used.sum()
    number = torch.arange(s["n_pages"], device=table.device)
    movers, holes = number[used & (number >= live)], number[~used & (number < live)]
    to = number.clone()
    to[movers] = holes
    s["table_out"].copy_(torch.where(table >= 0, to[table.clamp_min(0).long()], -1))
    s["refs_out"].copy_(refs)
    s["refs_out"][holes] = refs[movers]
    s["refs_out"][live:] = 0
    s["live"].copy_(live)
    for x in ("k8", "v8", "k_scale", "v_scale"):
        s[x][:, holes] = s[x][:, movers]
    return (s["table_out"], s["refs_out"], s["live"]) + _pool(s)


# ----------------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2607_21599_b200 import api

    Hq, Hkv = s["heads"]
    p = api.make_page_params(s["n_pages"], s["T"], Hkv, s["n_seqs"], s["max_pages"], n_layers=s["layers"])
    pool = (s["k8"], s["v8"], s["k_scale"], s["v_scale"])
    ws = s["workspace"]
    if s["kind"] == "write":
        api.check(api.daf_page_write(p, 0, s["n"], None, s["lens"], s["row_off"], s["idx"], s["max_rows"], s["k"], s["v"],
                                     s["table"], s["refs"], *pool, ws))
        return _pool(s)
    if s["kind"] == "read":
        api.check(api.daf_page_read(p, 0, s["n"], None, None, s["row_off"], s["max_rows"], s["table"], *pool, s["k_rows"],
                                    s["v_rows"], ws))
        return s["k_rows"], s["v_rows"]
    if s["kind"] == "attn":
        api.check(api.daf_page_attn(p, 0, s["n"], None, s["lens"], s["q"].shape[1], Hq, 0.0, s["q"], s["table"], *pool,
                                    s["out"], s["lse"], ws))
        return s["out"], s["lse"]
    if s["kind"] == "fork":
        api.check(api.daf_page_free(p, s["n"], s["dst"], None, s["table"], s["refs"], ws))
        api.check(api.daf_page_fork(p, s["n"], s["src"], s["dst"], s["keep"], s["want"], s["share"], s["table"], s["refs"], *pool, ws))
        return (s["table"], s["refs"]) + _pool(s)
    api.check(api.daf_page_compact(p, s["table"], s["refs"], s["table_out"], s["refs_out"], s["live"], *pool, ws))
    return (s["table_out"], s["refs_out"], s["live"]) + _pool(s)


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "read": _plain_read, "attn": _plain_attn, "fork": _plain_fork,
            "compact": _plain_compact}[state["kind"]](state)


# -------------------------------------------------------------------------------------------------------------- 64 bits
def _value(bytes_):
    """What a byte stands for: 1 sign, 4 exponent (bias 7) and 3 mantissa bits."""
    b = bytes_.to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.double() - 10))
    return torch.where(b >= 128, -mag, mag)


def _round8(x):
    """The nearest of the values a byte can stand for, ties to the even one."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -40))).clamp_min(-6)
    e = torch.where(x.abs() >= torch.exp2(e + 1), e + 1, e)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_write(s):
    T, table = s["T"], s["table"].tolist()
    lens, off = s["lens"].tolist(), s["row_off"].tolist()
    out = []
    for x in "kv":
        val, scale = _value(s[x + "8"][0]), s[x + "_scale"][0].double().clone()
        for b, L in enumerate(lens):
            rows = s[x][off[b]:off[b + 1]].double()
            pos = s["idx"].tolist() if s["idx"] is not None else list(range(L - len(rows), L))
            kept_to = L if s["idx"] is not None else L - len(rows)
            here = {}
            for i, at in enumerate(pos):
                here.setdefault(at // T, []).append((i, at % T))
            for j, put in here.items():
                pg = table[b][j]
                new = rows[[i for i, _ in put]]                                  # [m, Hkv, D]
                # (the logarithm of a power of two may come out a little above it; the next bf16 value is 2^-8 away)
                need = torch.exp2(torch.ceil(torch.log2(new.abs().amax((0, 2)) / 448) - 1e-9)).clamp_min(MIN_SCALE)
                taken = {t for _, t in put}
                kept = [t for t in range(T) if j * T + t < kept_to and t not in taken]
                to = torch.maximum(need, scale[pg]) if kept else need
                if kept:
                    val[pg][:, kept] = _round8(val[pg][:, kept] * (scale[pg] / to)[:, None, None])
                val[pg][:, [t for _, t in put]] = _round8(new.transpose(0, 1) / to[:, None, None])
                scale[pg] = to
        out.append((val[None], scale[None]))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def _exact_attn(s):
    (Hq, Hkv), T = s["heads"], s["T"]
    n, L_q = s["q"].shape[:2]
    out = torch.zeros(n, L_q, Hq, D, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((n, Hq, L_q), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, L in enumerate(s["lens"].tolist()):
        pages = s["table"][b, :_pages(L, T)].long()
        for h in range(Hkv):
            k, v = [(_value(s[x + "8"][0][pages, h]) * s[x + "_scale"][0][pages, h].double()[:, None, None]).reshape(-1, D)[:L] for x in "kv"]
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            for t in range(L_q):
                sees = L - L_q + t + 1
                if sees > 0:
                    z = s["q"][b, t, heads].double() @ k[:sees].T / math.sqrt(D)
                    lse[b, heads, t] = torch.logsumexp(z, -1)
                    out[b, t, heads] = torch.softmax(z, -1) @ v[:sees]
    return out, lse


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None                    # whole numbers, and bytes that move
    s = prepare(case, seed)
    if case["kind"] == "write":
        return _exact_write(s)
    if case["kind"] == "attn":
        return _exact_attn(s)
    rows = []
    for x in "kv":
        pages = s["table"][0].long()[:_pages(s["max_len"], s["T"])]
        wide = _value(s[x + "8"][0][pages]) * s[x + "_scale"][0][pages].double()[:, :, None, None]
        rows.append(torch.cat(list(wide.permute(0, 2, 1, 3)))[:s["max_len"]])
    return tuple(rows)
