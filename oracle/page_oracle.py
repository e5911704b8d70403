"""fp64 CPU definition of the paged 8-bit cache (the daf_page_* calls), in numpy and plain loops.

Test infrastructure: shares nothing with the CUDA code.  Pool arrays are [n_layers, n_pages, n_kv_heads, page_tokens, 128] uint8
with scales [n_layers, n_pages, n_kv_heads] float32, the table [n_seqs, max_pages] int32 and refs [n_pages] int32.
"""
from __future__ import annotations

import math

import numpy as np

MIN_SCALE_EXP = -60


def _byte_values() -> np.ndarray:
    """What each of the 256 bytes stands for: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        mag = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[b] = math.nan if b & 127 == 127 else (-mag if b & 128 else mag)
    return v


VALUES = _byte_values()
_POSITIVE = VALUES[:127]                # ascending: 0, 2^-9, ..., 448


def encode(x: np.ndarray) -> np.ndarray:
    """The byte nearest to each value (ties to the even byte, magnitudes over 448 to 448, NaN to 0x7f)."""
    x = np.asarray(x, np.float64)
    mag = np.minimum(np.abs(x), 448.0)
    hi = np.minimum(np.searchsorted(_POSITIVE, np.where(np.isnan(mag), 0.0, mag), side="left"), 126)
    lo = np.maximum(hi - 1, 0)
    d_hi, d_lo = _POSITIVE[hi] - mag, mag - _POSITIVE[lo]
    pick = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    out = pick | np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 127, out).astype(np.uint8)


def scale_exp(rows: np.ndarray) -> int:
    """Exponent of the least power of two that brings the finite values into the format's range, at least -60."""
    fin = np.abs(rows[np.isfinite(rows)])
    top = float(fin.max()) if fin.size else 0.0
    k = MIN_SCALE_EXP
    while top > 448.0 * 2.0 ** k:
        k += 1
    return k


def write(k8, scale, layer, seqs, lens, row_off, idx, rows, table, refs=None) -> None:
    """daf_page_write of one of K and V, in place."""
    T, H = k8.shape[3], k8.shape[2]
    rows = np.asarray(rows, np.float64)
    for b in range(len(lens)):
        seq = b if seqs is None else int(seqs[b])
        mine = range(int(row_off[b]), int(row_off[b + 1]))
        L, n = int(lens[b]), len(mine)
        place = {}
        for i, r in enumerate(mine):
            place[int(idx[r]) if idx is not None else L - n + i] = r      # of equal positions the last counts
        kept_to = L if idx is not None else L - n
        for j in sorted({p // T for p in place}):
            pg = int(table[seq, j])
            if not 0 <= pg < k8.shape[1] or (refs is not None and refs[pg] != 1):
                continue
            put = [(p - j * T, r) for p, r in place.items() if p // T == j]
            kept = [t for t in range(T) if j * T + t < kept_to and j * T + t not in place]
            for h in range(H):
                e = scale_exp(rows[[r for _, r in put], h])
                old = float(scale[layer, pg, h])
                if kept:
                    e = max(e, math.ceil(math.log2(old)))
                    if 2.0 ** e != old:
                        k8[layer, pg, h, kept] = encode(VALUES[k8[layer, pg, h, kept]] * (old / 2.0 ** e))
                for t, r in put:
                    k8[layer, pg, h, t] = encode(rows[r, h] / 2.0 ** e)
                scale[layer, pg, h] = 2.0 ** e


def bf16(x: np.ndarray) -> np.ndarray:
    """Rounds float32 to the nearest bf16 (ties to even), returned as float32; NaN stays NaN."""
    u = np.asarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


def values(k8, scale, layer, seq, n, table) -> np.ndarray:
    """The first n tokens of a sequence as fp64 [n, n_kv_heads, 128]; NaN rows where there is no page."""
    T, H = k8.shape[3], k8.shape[2]
    out = np.full((n, H, 128), np.nan)
    for t in range(n):
        pg = int(table[seq, t // T])
        if 0 <= pg < k8.shape[1]:
            out[t] = VALUES[k8[layer, pg, :, t % T]] * scale[layer, pg].astype(np.float64)[:, None]
    return out


def read(k8, scale, layer, seq, first, n, table) -> np.ndarray:
    """Tokens first .. first + n - 1 as bf16(scale * value)."""
    return bf16(values(k8, scale, layer, seq, first + n, table)[first:].astype(np.float32))


def attn(q, k, v, L, present=None, scale=1.0 / math.sqrt(128.0)):
    """One sequence: q [L_q, Hq, 128], k and v [L, Hkv, 128] (fp64), query token t sees keys j <= L - L_q + t that are `present`.
    Returns (out, lse [Hq, L_q], mean |V| under the same weights, largest sum |q||k| scale) in fp64."""
    L_q, Hq = q.shape[:2]
    G = Hq // k.shape[1] if k.shape[1] else 1
    out, mag = np.zeros((L_q, Hq, 128)), np.zeros((L_q, Hq, 128))
    lse, dots = np.full((Hq, L_q), -np.inf), np.zeros((L_q, Hq))
    present = np.ones(L, bool) if present is None else present
    for t in range(L_q):
        see = np.flatnonzero(present[:max(0, L - L_q + t + 1)])
        if not see.size:
            continue
        for h in range(Hq):
            kk, vv = k[see, h // G], v[see, h // G]
            with np.errstate(invalid="ignore"):
                z = (kk @ q[t, h]) * scale
                top = z.max()
                p = np.exp(z - top)
                lse[h, t] = top + math.log(p.sum()) if not np.isnan(p.sum()) else np.nan
                p /= p.sum()
                out[t, h] = p @ vv
                mag[t, h] = p @ np.abs(vv)
                dots[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * scale
    return out, lse, mag, dots


class Pool:
    """Table, refs and page contents under fork, free and compact, one item after the other."""

    def __init__(self, table, refs, T, pools):
        self.table, self.refs, self.T, self.pools = table, refs, T, pools      # pools: arrays [n_layers, n_pages, ...]

    def fork(self, src, dst, keep, want, share) -> str:
        """'' when done, 'bounds' or 'pages' when refused (nothing is changed then)."""
        T, n_seqs, M, P = self.T, *self.table.shape, len(self.refs)
        for i, (s, d) in enumerate(zip(src, dst)):
            kp = keep[i] if s >= 0 else 0
            if not 0 <= d < n_seqs or s >= n_seqs or not 0 <= want[i] <= M * T or not 0 <= kp <= M * T:
                return "bounds"
            if list(dst).count(d) > 1 or (s >= 0 and s != d and s in dst):
                return "bounds"
            held = -(-kp // T)
            have = int((self.table[d] >= 0).sum())
            if (s == d and held > have) or (s != d and have > 0) or (s >= 0 and s != d and not all(0 <= e < P for e in self.table[s, :held])):
                return "bounds"
            if s == d and kp // T < have and not 0 <= self.table[d, kp // T] < P:
                return "bounds"
        free = [p for p in range(P) if self.refs[p] == 0]
        refs0 = self.refs.copy()
        plan, used = [], 0
        for i, (s, d) in enumerate(zip(src, dst)):
            kp = keep[i] if s >= 0 else 0
            whole, held, pages = kp // T, -(-kp // T), -(-want[i] // T)
            row, copies = [-1] * M, []
            if s == d:
                row = self.table[d].tolist()
                have = sum(e >= 0 for e in row)
                if whole < have and refs0[row[whole]] > 1:      # the page that token `keep` goes into, with tokens of the row in it or not
                    copies.append((row[whole], whole))
                new = [c for _, c in copies] + list(range(have, pages))
            else:
                first = whole if share else 0
                if s >= 0:
                    row[:first] = self.table[s, :first].tolist()
                    copies = [(int(self.table[s, c]), c) for c in range(first, held)]
                new = list(range(first, max(pages, held)))
            plan.append((d, row, copies, new, s == d, used))
            used += len(new)
        if used > len(free):
            return "pages"
        for d, row, copies, new, grows, at in plan:
            if not grows:
                for e in row:
                    if e >= 0:
                        self.refs[e] += 1
            for i, c in enumerate(new):
                if row[c] >= 0:
                    self.refs[row[c]] -= 1
                row[c] = free[at + i]
                self.refs[row[c]] = 1
            self.table[d] = row
            for old, c in copies:
                for x in self.pools:
                    x[:, row[c]] = x[:, old]
        return ""

    def free(self, seqs, keep=None) -> None:
        for i, s in enumerate(seqs):
            held = -(-(0 if keep is None else keep[i]) // self.T)
            for c in range(held, self.table.shape[1]):
                if self.table[s, c] >= 0:
                    self.refs[self.table[s, c]] -= 1
                    self.table[s, c] = -1

    def compact(self) -> int:
        used = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        live = len(used)
        movers = [p for p in used if p >= live]
        holes = [p for p in range(live) if self.refs[p] == 0]
        to = dict(zip(movers, holes))
        for old, new in to.items():
            self.refs[new], self.refs[old] = self.refs[old], 0
            for x in self.pools:
                x[:, new] = x[:, old]
        for e in np.nditer(self.table, op_flags=["readwrite"]):
            if int(e) in to:
                e[...] = to[int(e)]
        return live
