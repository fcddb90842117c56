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

    def grow(self, slots, counts):
        slots = self._check_slots(slots)
        need = []
        for s, c in zip(slots, counts):
            if c < 0 or self.lengths[s] + int(c) > self.max_pages * PAGE:
                raise Refused("length")
            need.append(pages_of(self.lengths[s] + c) - pages_of(self.lengths[s]))
        new = list(self._take(sum(need)))
        for s, c, k in zip(slots, counts, need):
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
