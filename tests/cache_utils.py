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


def attend_bound(q, v, codes, scale, out, p, softmax_scale, k=None):
    """How far a row of essa_cache_attend may be from the fp64 result, element by element; one entry, all heads.

    * out is rounded to bf16 once: 2^-8 |out|;
    * a weight times the value's scale is rounded to bf16 before it meets (code - 8): 2^-8 sum_k p_k s_k |c_k - 8|;
    * a score is wrong by at most `d` and moves the weights by a factor e^(+-2 d) at most: (e^(2 d) - 1) sum_k p_k |v_k|.  The tensor core adds
      64 products of q (128 + code) <= 143 |q| in fp32 (taken as 16 roundings of 2^-23), the scales and the second term
      (minimum - 128 scale) sum(q) come on top with 2^-22 of terms of the same size: d = scale * 2^-18 * 143 * sum_g max_k(s_g) sum|q_g|
      + 2^-21 max|score| for the final product and exponent (and, with k, the rounding of k to bf16 in the
      tile kernel: eight standard deviations of a sum of independent errors of at most 2^-8 |q_i k_i| each).
    * fp32 sums of weights: 2^-16 sum_k p_k |v_k|."""
    rows, heads, d = q.shape
    kvh = v.shape[0]
    group = heads // kvh
    tol = np.zeros_like(out)
    for h in range(heads):
        c = h // group
        centred = np.abs(codes[c, 1].astype(np.float64) - 8) * np.repeat(scale[c, 1].astype(np.float64), co.GROUP, -1)
        qa = np.abs(q[:, h].astype(np.float64))
        smax = scale[c, 0].astype(np.float64).max(0, initial=0.0)  # per group
        err = softmax_scale * 2.0 ** -18 * 143 * (qa.reshape(rows, -1, co.GROUP).sum(-1) * smax).sum(-1)
        if k is not None and k.shape[1]:
            e2 = np.max((qa ** 2) @ (np.abs(k[c]) ** 2).T, axis=1)
            err = err + softmax_scale * 8 * 2.0 ** -8 / np.sqrt(3) * np.sqrt(e2)
        big = np.max(np.abs(q[:, h].astype(np.float64) @ (k[c] if k is not None else v[c]).T), axis=1, initial=0.0) * softmax_scale
        err = err + 2.0 ** -21 * big
        spread = p[:, h] @ np.abs(v[c])
        tol[:, h] = 2.0 ** -8 * np.abs(out[:, h]) + 2.0 ** -8 * (p[:, h] @ centred) + (np.expm1(2 * err)[:, None] + 2.0 ** -16) * spread + 1e-30
    return tol
