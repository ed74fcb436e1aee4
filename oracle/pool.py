"""The 8-bit paged cache by its definitions, on the CPU: pages and counts one claim after another, entries one block of 16 positions
at a time, attention in fp64 one row at a time.  Written from the formulas of include/sjd.h's sjd_pool section, not from any kernel."""
from __future__ import annotations

import math

import numpy as np

PAGE, BLOCK = 64, 16


class Refused(Exception):
    pass


# ------------------------------------------------------------------------------------------------ numbers of eight bits
def _e4m3_table():
    """Value of every byte: sign, four bits of exponent (bias 7), three of mantissa; 0x7F and 0xFF are NaN."""
    out = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = (m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            v = math.nan
        out[b] = -v if b & 128 else v
    return out


E4M3 = _e4m3_table()
_POSITIVE = E4M3[:127]     # 0 .. 448, rising


def to_e4m3(x):
    """Bytes of the nearest numbers, ties to the even mantissa, beyond +-448 the largest; not finite: NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    byte = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(hi % 2 == 0, hi, lo)))
    byte = np.where(_POSITIVE[hi] == a, hi, byte)
    return np.where(np.isfinite(x), byte | (np.signbit(x).astype(np.int64) << 7), 0x7F).astype(np.uint8)


def clamp_exp(e):
    return np.clip(np.asarray(e, np.int64), -100, 100)


def block_exponent(rows):
    """Smallest e with every finite |entry| <= 448 * 2^e (0: all zero)."""
    a = np.abs(rows[np.isfinite(rows)])
    top = float(a.max()) if a.size else 0.0
    if top == 0.0:
        return 0
    f, e = math.frexp(top)           # top = f 2^e, 1/2 <= f < 1; 448 = 7/8 2^9
    return int(np.clip(e - 9 + (f > 0.875), -100, 100))


# ------------------------------------------------------------------------------------------------ rotary positions
def rope_axes(pairs, interleaved):
    """Axis of every pair."""
    if not interleaved:
        return [a for a, n in enumerate(pairs) for _ in range(n)]
    left, out = list(pairs), []
    while sum(left):
        for a in range(len(pairs)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return out


def rope_angles(pos, head_dim, pairs, theta=10000.0, interleaved=False, per_axis=False):
    """Angles [row][pair] in fp64 of positions [row][axis]."""
    axes, seen, out = rope_axes(pairs, interleaved), [0] * len(pairs), np.zeros((len(pos), head_dim // 2))
    for i, a in enumerate(axes):
        f = seen[a] / pairs[a] if per_axis else 2.0 * i / head_dim
        seen[a] += 1
        out[:, i] = np.asarray(pos)[:, a].astype(np.float64) * theta ** -f
    return out


def rotate(x, angles):
    """x [row][head][head_dim] fp32; cosine and sine rounded to fp32, every product and sum an fp32 operation."""
    half = x.shape[-1] // 2
    c, s = np.cos(angles).astype(np.float32)[:, None], np.sin(angles).astype(np.float32)[:, None]
    a, b = x[..., :half].astype(np.float32), x[..., half:].astype(np.float32)
    return np.concatenate((a * c - b * s, b * c + a * s), -1)


# ------------------------------------------------------------------------------------------------ the pool
class Pool:
    """bytes uint8 [n][layer][2][kvh][64][hd], exps int8 [n][layer][2][kvh][4], table int32 [seq][pages], refs int32 [n]."""

    def __init__(self, pages, exps, table, refs):
        self.pages, self.exps, self.table, self.refs = pages.copy(), exps.copy(), table.copy(), refs.copy()

    def _check_list(self, seqs):
        if len(set(seqs)) < len(seqs) or any(s < 0 or s >= len(self.table) for s in seqs):
            raise Refused

    def reserve(self, seqs, begin, end):
        self._check_list(seqs)
        per_seq = self.table.shape[1]
        if any(b < 0 or e > per_seq * PAGE or (e > b and b >= per_seq * PAGE) for b, e in zip(begin, end)):
            raise Refused
        table, refs, copies, given = self.table.copy(), self.refs.copy(), [], 0
        free = [int(i) for i in np.nonzero(refs == 0)[0]]
        for s, b, e in zip(seqs, begin, end):
            for at in (range(b // PAGE, (e - 1) // PAGE + 1) if e > b else ()):
                page = int(table[s, at])
                if page >= 0 and refs[page] == 1:
                    continue
                if given == len(free):
                    raise Refused
                new, given = free[given], given + 1
                if page >= 0:
                    refs[page] -= 1
                    if at * PAGE < b:
                        copies.append((page, new))
                refs[new] = 1
                table[s, at] = new
        for src, dst in copies:
            self.pages[dst], self.exps[dst] = self.pages[src], self.exps[src]
        self.table, self.refs = table, refs

    def fork(self, src, dst, length):
        self._check_list(dst)
        for s, d, n in zip(src, dst, length):
            k = -(-n // PAGE)
            if s < 0 or s >= len(self.table) or s in dst or n < 0 or k > self.table.shape[1] or (self.table[s, :k] < 0).any() \
                    or (self.table[d] != -1).any():
                raise Refused
        for s, d, n in zip(src, dst, length):
            for at in range(-(-n // PAGE)):
                self.table[d, at] = self.table[s, at]
                self.refs[self.table[s, at]] += 1

    def free(self, seqs, keep):
        self._check_list(seqs)
        if any(k < 0 for k in keep):
            raise Refused
        for s, k in zip(seqs, keep):
            for at in range(-(-k // PAGE), self.table.shape[1]):
                if self.table[s, at] >= 0:
                    self.refs[self.table[s, at]] -= 1
                    self.table[s, at] = -1

    def compact(self):
        used = [int(i) for i in np.nonzero(self.refs > 0)[0]]
        n = len(used)
        holes = [i for i in range(n) if self.refs[i] == 0]
        for src, dst in zip([i for i in used if i >= n], holes):
            self.pages[dst], self.exps[dst] = self.pages[src], self.exps[src]
            self.refs[dst], self.refs[src] = self.refs[src], 0
            self.table[self.table == src] = dst

    def append(self, layer, seq, start, k, v):
        """Rotated keys and values [row][kvh][hd] (fp32) of positions start ..: entries and exponents of every block they touch."""
        n = len(k)
        for base in range(start // BLOCK * BLOCK, start + n, BLOCK):
            page, blk = int(self.table[seq, base // PAGE]), base % PAGE // BLOCK
            kept, last = max(0, start - base), min(BLOCK, start + n - base)
            for which, x in enumerate((k, v)):
                for h in range(k.shape[1]):
                    plane = self.pages[page, layer, which, h, blk * BLOCK:(blk + 1) * BLOCK]
                    e_old = int(clamp_exp(self.exps[page, layer, which, h, blk]))
                    rows = np.concatenate((E4M3[plane[:kept]] * 2.0 ** e_old, x[base + kept - start:base + last - start, h].astype(np.float64)))
                    e = block_exponent(rows)
                    plane[:last] = to_e4m3(rows * 2.0 ** -e)
                    self.exps[page, layer, which, h, blk] = e

    def entries(self, layer, seq, which, h, n):
        """The first n keys (0) or values (1) of a head: e4m3 numbers [n][hd] and their factors [n][1], fp64."""
        pages = self.table[seq, :-(-n // PAGE)]
        raw = E4M3[self.pages[pages, layer, which, h]].reshape(-1, self.pages.shape[-1])
        return raw[:n], 2.0 ** clamp_exp(self.exps[pages, layer, which, h]).reshape(-1).repeat(BLOCK)[:n, None]

    def attention(self, layer, q, seqs, in_pos, window, sliding=0, sinks=0, scale=None):
        """fp64 [row][head][hd] of q [row][head][hd], and what tolerances are made of:
        mass   sum_j p_j |v_j|
        floor  max_j (p_j 2^e_j) sum_j |e4m3 number of v_j|
        reach  max_j scale sum |q||k_j|
        flat   max_j scale max|q| sum |k_j|"""
        m, heads, hd = q.shape
        kvh = self.pages.shape[3]
        scale = hd ** -0.5 if not scale else float(scale)
        out, mass, floor = (np.zeros((m, heads, hd)) for _ in range(3))
        reach, flat = np.zeros((m, heads)), np.zeros((m, heads))
        for b, seq in enumerate(seqs):
            pos = np.asarray(in_pos[b * window:(b + 1) * window])
            n = int(pos.max()) + 1
            if n < 1:
                continue
            j = np.arange(n)
            for h in range(kvh):
                (k, ke), (v, ve) = self.entries(layer, seq, 0, h, n), self.entries(layer, seq, 1, h, n)
                k = k * ke
                for w in range(window):
                    seen = (j <= pos[w]) & ((sliding == 0) | (j > pos[w] - sliding) | (j < sinks))
                    if not seen.any():
                        continue
                    ks, vs, es = k[seen], v[seen], ve[seen]
                    at = b * window + w, slice(h * heads // kvh, (h + 1) * heads // kvh)
                    x = q[at].astype(np.float64)
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = scale * (x @ ks.T)
                        p = np.exp(s - s.max(-1, keepdims=True))
                        p = p / p.sum(-1, keepdims=True) * es[:, 0]
                        out[at], mass[at] = p @ vs, p @ np.abs(vs)
                        floor[at] = p.max(-1, keepdims=True) * np.abs(vs).sum(0)
                        reach[at] = scale * (np.abs(x) @ np.abs(ks).T).max(-1)
                        flat[at] = scale * np.abs(x).max(-1) * np.abs(ks).sum(-1).max()
        return out, mass, floor, reach, flat
