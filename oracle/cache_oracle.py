"""Plain, slow fp64 / integer model of the paged 4-bit key / value cache (numpy), written from include/essa.h.

Shares no code with csrc/.  Values are kept per (layer, page, kv head, K or V, token): codes, scale and minimum; the byte
layout of a page is produced and parsed separately, so that a test can compare bytes and values independently.
"""
from __future__ import annotations

import numpy as np

PAGE = 64
GROUP = 64


def quantize(x):
    """x [..., d] (bf16-representable, any float type): codes uint8 [..., d], scale and minimum fp16 [..., d / 64].

    minimum = fp16(min), scale = fp16((max - minimum) / 15), code = rint((x - minimum) / scale) clipped to 0 .. 15."""
    g = np.asarray(x, np.float32).reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(all="ignore"):
        low = g.min(-1).astype(np.float16)
        base = low.astype(np.float32)
        scale = ((g.max(-1) - base) / np.float32(15)).astype(np.float16)
        s = scale.astype(np.float32)
        code = np.rint((g - base[..., None]) / np.where(s > 0, s, 1)[..., None])
        code = np.where(s[..., None] > 0, np.clip(np.nan_to_num(code), 0, 15), 0).astype(np.uint8)
    return code.reshape(x.shape), scale, low


def quantize_tokens(k, v):
    """Both halves of tokens [T, kv_heads, d]; a token whose keys or values do not fit has keys of NaN and values of 0."""
    out = []
    bad = np.zeros(k.shape[:-1], bool)
    for x in (k, v):
        codes, scale, low = quantize(x)
        bad |= ~(np.isfinite(x).all(-1) & np.isfinite(scale).all(-1) & np.isfinite(low).all(-1))
        out.append([codes, scale, low])
    for (codes, scale, low), stored in zip(out, (np.nan, 0)):
        codes[bad], scale[bad], low[bad] = 0, 0, stored
    return out


def dequantize(codes, scale, low):
    g = codes.reshape(*codes.shape[:-1], codes.shape[-1] // GROUP, GROUP).astype(np.float64)
    return (g * scale.astype(np.float64)[..., None] + low.astype(np.float64)[..., None]).reshape(codes.shape)


def pages_of(tokens):
    return -(-int(tokens) // PAGE)


class Refused(Exception):
    """The call changes nothing and ESSA_ERR_CACHE is recorded."""


class Cache:
    """Page management on integers, storage on (codes, scale, minimum) arrays."""

    def __init__(self, layers, num_pages, kv_heads, head_dim, max_seqs, max_pages):
        self.shape = (layers, num_pages, kv_heads, head_dim)
        self.max_seqs, self.max_pages, self.num_pages = max_seqs, max_pages, num_pages
        self.table = np.full((max_seqs, max_pages), -1, np.int32)
        self.lengths = np.zeros(max_seqs, np.int32)
        self.refs = np.zeros(num_pages, np.int32)
        self.codes = np.zeros((layers, num_pages, kv_heads, 2, PAGE, head_dim), np.uint8)
        self.scale = np.zeros((layers, num_pages, kv_heads, 2, PAGE, head_dim // GROUP), np.float16)
        self.low = np.zeros_like(self.scale)

    # -- bytes
    def load_bytes(self, raw):
        layers, pages, heads, d = self.shape
        b = raw.reshape(layers, pages, heads, 72 * d)
        code = b[..., :64 * d].reshape(layers, pages, heads, 2, d // 32, PAGE, 16)
        for c in range(d):
            self.codes[..., c] = (code[..., c // 32, :, (c % 32) // 2] >> (4 * (c % 2))) & 15
        meta = np.ascontiguousarray(b[..., 64 * d:]).view(np.float16).reshape(layers, pages, heads, 2, d // GROUP, PAGE, 2)
        self.scale[:] = np.moveaxis(meta[..., 0], -2, -1)
        self.low[:] = np.moveaxis(meta[..., 1], -2, -1)

    def to_bytes(self):
        layers, pages, heads, d = self.shape
        code = np.zeros((layers, pages, heads, 2, d // 32, PAGE, 16), np.uint8)
        for c in range(d):
            code[..., c // 32, :, (c % 32) // 2] |= self.codes[..., c] << (4 * (c % 2))
        meta = np.stack([np.moveaxis(self.scale, -1, -2), np.moveaxis(self.low, -1, -2)], -1)
        lead = (layers, pages, heads)
        return np.concatenate([code.reshape(*lead, -1), np.ascontiguousarray(meta).view(np.uint8).reshape(*lead, -1)], -1).reshape(layers, pages, -1)

    # -- pages
    def _take(self, n):
        free = np.flatnonzero(self.refs == 0)
        if len(free) < n:
            raise Refused("too few free pages")
        return free[:n]

    def _check_slots(self, slots):
        slots = [int(s) for s in slots]
        if any(s < 0 or s >= self.max_seqs for s in slots) or len(set(slots)) < len(slots):
            raise Refused("bad slots")
        return slots

    def _drop(self, s):
        for p in self.table[s]:
            if p >= 0:
                self.refs[p] -= 1
        self.table[s] = -1
        self.lengths[s] = 0

    def _shared_end(self, s):
        """The page that sequence s ends in the middle of and that another one shares; None: it does not."""
        n = int(self.lengths[s])
        p = int(self.table[s, n // PAGE]) if n % PAGE else -1
        return p if 0 <= p < self.num_pages and self.refs[p] > 1 else None

    def grow(self, slots, counts):
        slots = self._check_slots(slots)
        need, ends = [], []
        for s, c in zip(slots, counts):
            if c < 0 or self.lengths[s] + int(c) > self.max_pages * PAGE:
                raise Refused("length")
            need.append(pages_of(self.lengths[s] + c) - pages_of(self.lengths[s]))
            ends.append(self._shared_end(s) if c > 0 else None)
        new = list(self._take(sum(need) + sum(e is not None for e in ends)))
        for s, c, k, old in zip(slots, counts, need, ends):
            if old is not None:
                p = new.pop(0)
                for a in (self.codes, self.scale, self.low):
                    a[:, p] = a[:, old]
                self.table[s, self.lengths[s] // PAGE] = p
                self.refs[p] = 1
                self.refs[old] -= 1
            at = pages_of(self.lengths[s])
            for j in range(k):
                p = new.pop(0)
                self.table[s, at + j] = p
                self.refs[p] = 1
            self.lengths[s] += c

    def free(self, slots):
        for s in self._check_slots(slots):
            self._drop(s)

    def fork(self, src, dst, lens=None):
        dst = self._check_slots(dst)
        src = [int(s) for s in src]
        if any(s < 0 or s >= self.max_seqs or s in dst for s in src):
            raise Refused("bad src")
        lens = [int(self.lengths[s]) for s in src] if lens is None else [int(x) for x in lens]
        if any(x < 0 or x > self.lengths[s] for s, x in zip(src, lens)):
            raise Refused("length")
        before = self.table.copy(), self.lengths.copy(), self.refs.copy()
        for d in dst:
            self._drop(d)
        try:
            new = list(self._take(sum(x % PAGE > 0 for x in lens)))
        except Refused:
            self.table, self.lengths, self.refs = before
            raise
        for s, d, x in zip(src, dst, lens):
            full = x // PAGE
            self.table[d, :full] = self.table[s, :full]
            if x % PAGE:
                p, old = new.pop(0), self.table[s, full]
                self.table[d, full] = p
                for a in (self.codes, self.scale, self.low):
                    a[:, p] = a[:, old]
            for p in self.table[d]:
                if p >= 0:
                    self.refs[p] += 1
            self.lengths[d] = x

    def compact(self):
        used = np.flatnonzero(self.refs > 0)
        n = len(used)
        movers, holes = used[used >= n], [p for p in range(n) if self.refs[p] == 0]
        to = np.arange(self.num_pages)
        for old, new in zip(movers, holes):
            to[old] = new
            for a in (self.codes, self.scale, self.low):
                a[:, new] = a[:, old]
            self.refs[new], self.refs[old] = self.refs[old], 0
        self.table = np.where(self.table >= 0, to[np.maximum(self.table, 0)], -1).astype(np.int32)
        return n

    # -- tokens
    def append(self, layer, k, v, offsets, slots):
        (kc, ks, kl), (vc, vs, vl) = quantize_tokens(k, v)
        for i, s in enumerate(slots):
            rows = offsets[i + 1] - offsets[i]
            for j in range(rows):
                pos, t = self.lengths[s] - rows + j, offsets[i] + j
                p = self.table[s, pos // PAGE]
                for a, new in ((self.codes, (kc, vc)), (self.scale, (ks, vs)), (self.low, (kl, vl))):
                    a[layer, p, :, 0, pos % PAGE] = new[0][t]
                    a[layer, p, :, 1, pos % PAGE] = new[1][t]

    def sequence(self, layer, s):
        """(K, V) [kv_heads, length, d] fp64 of sequence s, and their codes and scales [kv_heads, 2, length, ...]."""
        ids = [int(p) for p in self.table[s, :pages_of(self.lengths[s])]]
        cat = lambda a: np.concatenate([a[layer, p] for p in ids], axis=2)[:, :, :self.lengths[s]] if ids else a[layer, 0][:, :, :0]
        codes, scale, low = cat(self.codes), cat(self.scale), cat(self.low)
        x = dequantize(codes, scale, low)
        return x[:, 0], x[:, 1], codes, scale


def attend(q, k, v, length, scale):
    """q [rows, heads, d], k, v [kv_heads, length, d] fp64; row j is token length - rows + j.  (out, p): p [rows, heads, length]."""
    rows, heads, d = q.shape
    group = heads // k.shape[0]
    out, weights = np.zeros((rows, heads, d)), np.zeros((rows, heads, length))
    for j in range(rows):
        see = length - rows + j + 1
        if see <= 0:
            continue
        for h in range(heads):
            s = k[h // group, :see] @ q[j, h].astype(np.float64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            weights[j, h, :see] = p
            out[j, h] = p @ v[h // group, :see]
    return out, weights


# -- masks, trees, rotation
def attend_seen(q, k, v, seen, scale):
    """q [rows, heads, d], k, v [kv_heads, length, d] fp64, seen [rows, length]: (out, p) as attend; a row that sees nothing is 0."""
    rows, heads, d = q.shape
    group = heads // k.shape[0]
    out, weights = np.zeros((rows, heads, d)), np.zeros((rows, heads, k.shape[1]))
    for j in range(rows):
        at = np.flatnonzero(seen[j])
        if not len(at):
            continue
        for h in range(heads):
            s = k[h // group, at] @ q[j, h].astype(np.float64) * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            weights[j, h, at] = p
            out[j, h] = p @ v[h // group, at]
    return out, weights


def seen_mask(length, rows, window=None, sinks=0, drafts=None):
    """[rows, length]: what the last `rows` tokens of a sequence see.  window, sinks as in essa_attend_mask; drafts [rows, rows] bool: which draft sees which."""
    past = length - rows
    seen = np.zeros((rows, length), bool)
    for j in range(rows):
        pos = past + (j if drafts is None else int(drafts[j].sum()) - 1)
        for s in range(length):
            known = s <= pos if drafts is None else s < past
            near = window is None or s > pos - window or s < sinks
            seen[j, s] = known and near
            if drafts is not None and s >= past:
                seen[j, s] = drafts[j, s - past]
    return seen


def ancestors(parents):
    """(bits [n, n] bool, depth [n]) of drafted tokens; a parent that is not before its child counts as -1."""
    n = len(parents)
    bits, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
    for j in range(n):
        at, depth[j] = j, -1
        while at >= 0:
            bits[j, at] = True
            depth[j] += 1
            at = parents[at] if -1 <= parents[at] < at else -1
    return bits, depth


def pack_bits(bits, words):
    """[n, n] bool -> [n, words] uint32, bit j % 32 of word j / 32."""
    out = np.zeros((len(bits), words), np.uint32)
    for r, row in enumerate(bits):
        for j in np.flatnonzero(row[:32 * words]):
            out[r, j // 32] |= np.uint32(1 << (int(j) % 32))
    return out


def keep(cache, slots, rows, counts, picks=None):
    """essa_cache_keep on a Cache: of the last rows[i] tokens of slots[i], picks[i][:counts[i]] (None: the first) stay."""
    slots = cache._check_slots(slots)
    for i, s in enumerate(slots):
        length, L, c = int(cache.lengths[s]), int(rows[i]), int(counts[i])
        if not (0 <= L <= length and 0 <= c <= L):
            raise Refused("length")
        mine = list(range(c)) if picks is None else [int(x) for x in picks[i][:c]]
        if picks is not None and (L > 256 or c > len(picks[i]) or any(b <= a for a, b in zip(mine, mine[1:])) or any(p < 0 or p >= L for p in mine)):
            raise Refused("picks")
        base = length - L
        for j in range(base // PAGE, pages_of(length)):
            p = int(cache.table[s, j])
            if not 0 <= p < cache.num_pages or cache.refs[p] <= 0:
                raise Refused("page")
        moved = [m for m, p in enumerate(mine) if p != m]
        if moved:
            for j in range((base + moved[0]) // PAGE, (base + c - 1) // PAGE + 1):
                if cache.refs[cache.table[s, j]] != 1:
                    raise Refused("shared")
    for i, s in enumerate(slots):
        length, L, c = int(cache.lengths[s]), int(rows[i]), int(counts[i])
        base = length - L
        at = lambda t: (int(cache.table[s, t // PAGE]), t % PAGE)
        for m, p in enumerate([] if picks is None else picks[i][:c]):
            (p0, o0), (p1, o1) = at(base + int(p)), at(base + m)
            for a in (cache.codes, cache.scale, cache.low):
                a[:, p1, :, :, o1] = a[:, p0, :, :, o0]
        for j in range(pages_of(base + c), pages_of(length)):
            cache.refs[cache.table[s, j]] -= 1
            cache.table[s, j] = -1
        cache.lengths[s] = base + c


def rotate(x, positions, frequencies, axis, adjacent=False, magnitude=1.0):
    """x [T, heads, d], positions [axes, T]: fp64, angles modulo a turn in exact rational arithmetic of the fp64 frequencies (2 pi to 50 digits)."""
    from fractions import Fraction
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021")
    T, heads, d = x.shape
    half = d // 2
    y, out = x.astype(np.float64), np.zeros(x.shape)
    for i in range(half):
        turn = Fraction(float(frequencies[i])) / two_pi
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        for t in range(T):
            part = turn * int(positions[axis[i]][t])
            angle = 2 * np.pi * float(part - (part.numerator // part.denominator))
            c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
            out[t, :, a] = y[t, :, a] * c - y[t, :, b] * s
            out[t, :, b] = y[t, :, b] * c + y[t, :, a] * s
    return out
