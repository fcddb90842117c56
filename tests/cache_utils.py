"""Helpers of the cache tests: a cache on the GPU and its oracle side by side."""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle as co
from paper_2507_04453_b200 import workloads as wl


def bf16(rng, shape, scale=1.0):
    return wl.round_to_bf16((rng.standard_normal(shape) * scale).astype(np.float32))


class Pair:
    """One cache: `gpu` (binding.KvCache) and `cpu` (oracle), set to the same state."""

    def __init__(self, torch, ctx, layers, num_pages, kv_heads, head_dim, max_seqs, max_pages):
        self.torch = torch
        self.gpu = ctx.kv_cache(layers, num_pages, kv_heads, head_dim, max_seqs, max_pages)
        self.cpu = co.Cache(layers, num_pages, kv_heads, head_dim, max_seqs, max_pages)
        self.gpu.pages.fill_(0xff)  # stale NaN scales and minima wherever nothing has been stored
        self.cpu.load_bytes(self.gpu.pages.cpu().numpy())

    def ints(self, a):
        return None if a is None else self.torch.tensor(np.asarray(a), dtype=self.torch.int32, device="cuda").reshape(-1)

    def bf(self, a):
        return self.torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(self.torch.bfloat16).cuda()

    def place(self, lengths, rng, shared=0):
        """Sequences of these lengths on pages in random order (the first `shared` pages of all sequences the same), random contents."""
        c = self.cpu
        need = [co.pages_of(n) for n in lengths]
        order = list(rng.permutation(c.num_pages))
        common = [order.pop() for _ in range(shared)]
        for s, n in enumerate(lengths):
            k = min(need[s], shared) if n >= shared * co.PAGE else 0
            c.table[s, :need[s]] = common[:k] + [order.pop() for _ in range(need[s] - k)]
            c.lengths[s] = n
        for p in c.table[c.table >= 0]:
            c.refs[p] += 1
        live = sorted({int(p) for p in c.table[c.table >= 0]})
        if live:
            layers, _, heads, d = c.shape
            for layer in range(layers):
                x = bf16(rng, (2, len(live), co.PAGE, heads, d))
                for half in range(2):
                    codes, scale, low = co.quantize(x[half])
                    for a, new in ((c.codes, codes), (c.scale, scale), (c.low, low)):
                        a[layer, live, :, half] = np.swapaxes(new, 1, 2)
            # what lies behind a sequence's end in its last page stays as it is
            used = np.zeros((c.num_pages, co.PAGE), bool)
            for s, n in enumerate(lengths):
                for j in range(need[s]):
                    used[c.table[s, j], :min(co.PAGE, n - j * co.PAGE)] = True
            stale = ~used
            for a, val in ((c.codes, 15), (c.scale, np.nan), (c.low, np.nan)):
                np.moveaxis(a, 4, 2)[:, stale] = val
        self.push()

    def push(self):
        t = self.torch
        self.gpu.pages.copy_(t.from_numpy(self.cpu.to_bytes()))
        for name in ("table", "lengths", "refs"):
            getattr(self.gpu, name).copy_(t.from_numpy(getattr(self.cpu, name)))

    def assert_same(self, pages=True):
        self.torch.cuda.synchronize()
        for name in ("table", "lengths", "refs"):
            np.testing.assert_array_equal(getattr(self.gpu, name).cpu().numpy(), getattr(self.cpu, name), err_msg=name)
        if pages:
            got, want = self.gpu.pages.cpu().numpy(), self.cpu.to_bytes()
            # NaN minima compare by meaning, everything else by bits
            other = co.Cache(*self.cpu.shape, 1, 1)
            other.load_bytes(got)
            np.testing.assert_array_equal(other.codes, self.cpu.codes)
            np.testing.assert_array_equal(other.scale, self.cpu.scale)
            np.testing.assert_array_equal(other.low, self.cpu.low)
            assert got.shape == want.shape


def attend_bound(q, v, codes, scale, out, p, softmax_scale, k):
    """How far a row of essa_cache_attend may be from the fp64 result, element by element; one entry, all heads.  It holds for both kernels.

    * out is rounded to bf16 once: 2^-8 |out|;
    * few rows: a weight times the value's scale is rounded to fp16 before it meets (code - 8): 2^-11 sum_k p_k s_k |c_k - 8|, and where the
      product is 2^-14 below the unit (at most twice the largest scale of a group; the weights' sum is at least 1) 2^-24 max(s) absolutely;
      many rows: V and P are fp16, V's offset (minimum + 8 scale) too: 2^-11 sum_k p_k (2 |v_k| + |offset_k|), weights below
      2^-14 of the largest to 2^-25 absolutely: 2^-25 sum_k |v_k|;
    * a score is wrong by at most `err` and moves the weights by a factor e^(+-2 err) at most: (e^(2 err) - 1) sum_k p_k |v_k|.  Few rows: the
      tensor core adds 64 products of q (1024 + code), or q / 16 (1024 + 16 code), at most 1039 |q| each, in fp32 (taken as 16 roundings of
      2^-23); the scales and the second term minimum sum(q) come on top with 2^-22 of terms of the same size: scale * 2^-18 * 1039 *
      sum_g max_k(s_g) sum|q_g|, and 2^-21 max|score| for the final product and exponent.  Many rows: K is (code - 8) scale + offset
      with the offset and the result rounded to fp16: 2^-11 |offset| |sum q| per group, as it is the same for the whole group, and
      eight standard deviations of a sum of independent errors of at most 2^-11 |q_i k_i| each;
    * fp32 sums of weights: 2^-16 sum_k p_k |v_k|."""
    rows, heads, d = q.shape
    group = heads // v.shape[0]
    q = q.astype(np.float64)
    tol = np.zeros_like(out)
    for h in range(heads):
        c = h // group
        s = scale[c].astype(np.float64)                                      # [2, keys, groups]
        centred = (codes[c].astype(np.float64) - 8) * np.repeat(s, co.GROUP, -1)
        offset = np.stack([k[c], v[c]]) - centred
        qh, vh = q[:, h], np.abs(v[c])
        err = softmax_scale * 2.0 ** -18 * 1039 * (np.abs(qh).reshape(rows, -1, co.GROUP).sum(-1) * s[0].max(0, initial=0.0)).sum(-1)
        err = err + 2.0 ** -21 * softmax_scale * np.max(np.abs(qh @ k[c].T), axis=1, initial=0.0)
        shared = sum(np.abs(qh[:, g:g + co.GROUP] @ offset[0][:, g:g + co.GROUP].T) for g in range(0, d, co.GROUP))
        alone = 8 / np.sqrt(3) * np.sqrt((qh ** 2) @ (k[c] ** 2).T)
        err = err + softmax_scale * 2.0 ** -11 * np.max(shared + alone, axis=1, initial=0.0)
        ph = p[:, h]
        tol[:, h] = (2.0 ** -8 * np.abs(out[:, h]) + 2.0 ** -11 * (ph @ np.abs(centred[1])) + 2.0 ** -11 * (ph @ (2 * vh + np.abs(offset[1])))
                     + 2.0 ** -24 * 8 * ((ph > 0).sum(-1) * s[1].max(initial=0.0))[:, None] + 2.0 ** -25 * (ph > 0).astype(float) @ vh + (np.expm1(2 * err)[:, None] + 2.0 ** -16) * (ph @ vh) + 1e-30)
    return tol


# How far a row of one head may be from the fp64 result by norm, for keys, values and queries without a common direction (N(0, 1) and the like)
# and scores of a few units.  out is rounded to bf16 once: 2^-8 of every element at most, so 2^-8 of the norm.  What else is rounded belongs to one
# key each (its weight, its value, its score: 2^-11 of them, scores of a few units to less than 2^-11) and is as independent from key to key as
# the keys' contributions to the result are: whatever their number, sqrt(3) 2^-11 of the norm, taken as 2^-10.  Unlike attend_bound, which adds
# the worst cases, this does not grow with the number of keys: a page of 64 among n equal ones is sqrt(64 / n) of the norm.
NORM_LIMIT = 2.0 ** -8 + 2.0 ** -10


def norm_error(got, want):
    """|got - want| / |want| of every row and head; a row that sees nothing (want 0) has to be 0."""
    a, b = np.linalg.norm(got.astype(np.float64) - want, axis=-1), np.linalg.norm(want, axis=-1)
    return np.where(b > 0, a / np.where(b > 0, b, 1), np.where(a > 0, np.inf, 0.0))
