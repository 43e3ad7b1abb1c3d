"""Inputs and tolerances shared by the tests of the cache operators."""

import numpy as np
import torch

from oracle import bf16_bits_to_f64
from oracle.cache import attend, kv4_pack, kv4_unpack, visible_keys
from tests.gpu_helpers import to_dev, to_f64
from workloads import f32_to_bf16_bits


def normal_bits(rng, shape, scale=1.0):
    return f32_to_bf16_bits(scale * rng.standard_normal(shape, dtype=np.float32))


class Batch:
    """Sequences of given lengths in one layout (dense, packed, paged bf16, or kv4), with
    noise in every row and table entry that no sequence owns."""

    def __init__(self, lengths, H_Q, H_KV, layout, page=64, seed=0, max_pages=None):
        rng = np.random.default_rng(seed)
        self.lengths, self.layout, self.H_KV = list(lengths), layout, H_KV
        B = len(lengths)
        self.q = normal_bits(rng, (B, H_Q, 128), 2.0)
        self.L = max(lengths)
        self.rows = []   # cache rows of each sequence's keys
        if layout in ("paged", "kv4"):
            need = [-(-n // page) for n in lengths]
            num = sum(need) + 3
            order = rng.permutation(num)
            mp = max(max(need), 1) if max_pages is None else max_pages
            self.table = rng.integers(0, num, (B, mp)).astype(np.int32)
            at = 0
            for b, n in enumerate(need):
                self.table[b, :n] = order[at:at + n]
                at += n
                j = np.arange(lengths[b])
                self.rows.append(self.table[b, j // page].astype(np.int64) * page + j % page)
            shape = (num, page, H_KV, 128)
        elif layout == "packed":
            self.cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
            self.rows = [self.cu[b] + np.arange(n) for b, n in enumerate(lengths)]
            shape = (sum(lengths), H_KV, 128)
        else:
            self.rows = [b * self.L + np.arange(self.L) for b in range(B)]
            shape = (B, self.L, H_KV, 128)
        self.k, self.v = normal_bits(rng, shape), normal_bits(rng, shape)
        if layout == "kv4":
            self.cache = kv4_pack(self.k.reshape(-1, H_KV, 128), self.v.reshape(-1, H_KV, 128), page)

    def reference(self, window, sinks, scale=None):
        if self.layout == "kv4":
            k, v = kv4_unpack(self.cache)
        else:
            k, v = (bf16_bits_to_f64(x).reshape(-1, self.H_KV, 128) for x in (self.k, self.v))
        seen = [self.rows[b][visible_keys(n, window, sinks)] for b, n in enumerate(self.lengths)]
        return attend(bf16_bits_to_f64(self.q), [k[r] for r in seen], [v[r] for r in seen], scale)

    def hidden_rows(self, window, sinks):
        """Cache rows that no query sees."""
        n = self.k.reshape(-1, self.H_KV, 128).shape[0]
        seen = np.zeros(n, dtype=bool)
        for b, L in enumerate(self.lengths):
            seen[self.rows[b][visible_keys(L, window, sinks)]] = True
        return ~seen

    def call_window(self, da, window, sinks, lse=None, **kw):
        q = to_dev(self.q)
        k, v = kw.pop("kv", None) or (to_dev(self.k), to_dev(self.v))
        if self.layout == "packed":
            kw.update(cu_seqlens_k=torch.from_numpy(self.cu).cuda())
        elif self.layout == "paged":
            kw.update(block_table=torch.from_numpy(self.table).cuda(), seq_lens=self.seq_lens())
        return da.da_decode_attn_window(q, k, v, window, sinks, L_K_max=kw.pop("L", self.L), lse_out=lse, **kw)

    def call_kv4(self, da, window=0, sinks=0, lse=None, cache=None, **kw):
        cache = torch.from_numpy(self.cache).cuda() if cache is None else cache
        return da.da_decode_attn_kv4(to_dev(self.q), cache, torch.from_numpy(self.table).cuda(), self.seq_lens(),
                                     kw.pop("L", self.L), window, sinks, lse_out=lse, **kw)

    def seq_lens(self):
        return torch.tensor(self.lengths, dtype=torch.int32, device="cuda")


def new_lse(batch):
    return torch.full(batch.q.shape[:2], 7.0, dtype=torch.float32, device="cuda")


def check_attention(out, lse, ref, what):
    """Each probability is rounded to bf16 before the second product (off by at most
    2^-8 of itself, so the output by 2^-8 of the weighted mean of |v|) and the output
    once more; 32-bit sums of up to 2^15 terms of either sign and exponents of 128
    products add less than 2^-12 of the same mean.  lse is 32-bit throughout: scores
    of a few tens, 128 products each, 2^-13."""
    o, l, size = ref
    got = to_f64(out)
    assert np.all(np.isfinite(got)), f"{what}: non-finite output"
    tol = (2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * np.abs(o) * (1 + 2.0 ** -7) + 1e-30
    worst = np.max(np.abs(got - o) / tol)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the tolerance"
    if lse is not None:
        g = lse.cpu().numpy().astype(np.float64)
        fin = np.isfinite(l)
        assert np.array_equal(np.isneginf(g), ~fin), f"{what}: lse of empty rows"
        err = np.max(np.abs(g[fin] - l[fin]), initial=0.0)
        assert err <= 2.0 ** -13, f"{what}: lse off by {err:.2e}"
