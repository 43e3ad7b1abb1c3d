"""The attention weights of keys against the fp64 oracle."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import attend, key_weights
from tests.cache_helpers import Batch
from tests.gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu


class Weights(Batch):
    def __init__(self, lengths, H_Q, H_KV, page=64, seed=0, spare=7, **kw):
        super().__init__(lengths, H_Q, H_KV, "paged", page, seed, **kw)
        rng = np.random.default_rng(seed + 1)
        self.stride = self.L + spare
        self.old = rng.exponential(0.3, (len(lengths), H_KV, self.stride)).astype(np.float32)
        k = bf16_bits_to_f64(self.k).reshape(-1, H_KV, 128)
        self.ks = [k[r] for r in self.rows]
        self.lse = attend(bf16_bits_to_f64(self.q), self.ks, self.ks)[1].astype(np.float32)

    def check(self, got, decay, what, scale=None):
        want, tol = key_weights(bf16_bits_to_f64(self.q), self.ks, self.lse.astype(np.float64),
                                [self.old[b, :, :n].astype(np.float64) for b, n in enumerate(self.lengths)],
                                float(np.float32(decay)), scale)
        got = got.cpu().numpy()
        for b, n in enumerate(self.lengths):
            worst = np.max(np.abs(got[b, :, :n] - want[b]) / tol[b], initial=0.0)
            assert worst <= 1.0, f"{what}: sequence {b}: {worst:.3f} of the tolerance"
            assert np.array_equal(got[b, :, n:], self.old[b, :, n:]), f"{what}: entries past sequence {b}"

    def call(self, decay, out=None, L=None, old=None, **kw):
        old = torch.from_numpy(self.old).cuda() if old is None else old
        return da.da_add_key_weights(to_dev(self.q), to_dev(self.k), torch.from_numpy(self.table).cuda(), self.seq_lens(),
                                     torch.from_numpy(self.lse).cuda(), old, self.L if L is None else L, decay, out, **kw)


@pytest.mark.parametrize("H_Q,H_KV", [(8, 1), (1, 1), (64, 8), (40, 8), (16, 16), (32, 1), (34, 2), (64, 1), (128, 2),
                                      (130, 1), (6, 3)])
@pytest.mark.parametrize("page", [32, 96])
def test_heads(H_Q, H_KV, page):
    w = Weights([1, 0, 31, 32, 33, 200, 385], H_Q, H_KV, page, seed=H_Q)
    say(f"weights {H_Q}/{H_KV} page {page}")
    got = w.call(1.0)
    torch.cuda.synchronize()
    w.check(got, 1.0, f"{H_Q}/{H_KV}")


@pytest.mark.parametrize("decay", [0.0, 0.5, 0.98, 1.0])
@pytest.mark.parametrize("place", ["own", "other"])
def test_decay_and_places(decay, place):
    w = Weights([77, 513], 8, 2, seed=3)
    old = torch.from_numpy(w.old).cuda()
    out = None if place == "own" else old.clone()
    say(f"weights decay {decay} {place}")
    got = w.call(decay, out, old=old)
    torch.cuda.synchronize()
    assert got is (old if out is None else out)
    w.check(got, decay, f"decay {decay}")
    if out is not None:
        assert np.array_equal(old.cpu().numpy(), w.old)


def test_decay_zero_does_not_read():
    w = Weights([100], 8, 1, seed=4)
    old = torch.full((1, 1, w.stride), float("nan"), device="cuda")
    say("weights decay 0 over NaN")
    got = w.call(0.0, old=old)
    torch.cuda.synchronize()
    assert torch.isfinite(got[..., :100]).all() and torch.isnan(got[..., 100:]).all()
    w.old[...] = np.nan
    got = got.cpu().numpy()[0, :, :100]
    want, tol = key_weights(bf16_bits_to_f64(w.q), w.ks, w.lse.astype(np.float64), None, 0.0)
    assert np.max(np.abs(got - want[0]) / tol[0]) <= 1.0


@pytest.mark.parametrize("L", [4000, 20000])
def test_a_bound_above_the_lengths(L):
    w = Weights([700, 64, 2049], 8, 2, page=32, seed=5, spare=20000, max_pages=700)
    say(f"weights under L_K_max {L}")
    got = w.call(1.0, L=L)
    torch.cuda.synchronize()
    w.check(got, 1.0, f"L_K_max {L}")


def test_a_bound_below_the_lengths_cuts_them():
    w = Weights([700, 64, 300], 8, 2, seed=6)
    say("weights under a lower L_K_max")
    got = w.call(1.0, L=256)
    torch.cuda.synchronize()
    w.lengths = [256, 64, 256]
    w.ks = [k[:256] for k in w.ks]
    w.check(got, 1.0, "cut")


def test_many_tiles_a_workgroup():
    w = Weights([70001, 40000], 4, 1, page=32, seed=7)
    say("weights of 70001 keys")
    got = w.call(0.5)
    torch.cuda.synchronize()
    w.check(got, 0.5, "70001 keys")


def test_scale_and_sums_over_a_step():
    w = Weights([333], 64, 8, seed=8)
    k = bf16_bits_to_f64(w.k).reshape(-1, 8, 128)
    w.lse = attend(bf16_bits_to_f64(w.q), [k[w.rows[0]]], [k[w.rows[0]]], 0.2)[1].astype(np.float32)
    say("weights scale 0.2")
    got = w.call(0.0, softmax_scale=0.2)
    torch.cuda.synchronize()
    w.check(got, 0.0, "scale", scale=float(np.float32(0.2)))
    # a softmax's weights sum to one a head: eight heads a KV head
    assert torch.allclose(got[0, :, :333].sum(dim=1), torch.full((8,), 8.0, device="cuda"), atol=1e-4)


def test_nothing_seen_bad_pages_and_what_is_not_finite():
    w = Weights([200, 96, 64], 24, 2, page=32, seed=9)
    w.lse[0, 3] = -np.inf           # a head that saw nothing adds nothing
    w.table[1, 1], w.table[1, 2] = -1, 10 ** 6   # zero keys
    kb = w.k.reshape(-1, 2, 128)
    w.ks[1] = w.ks[1].copy()
    w.ks[1][32:] = 0.0
    kb[w.rows[2][5], 0, 7] = 0x7FC0  # NaN in one key of one head
    kb[w.rows[2][6], 1, 3] = 0xFF80  # -inf: every score +-inf
    q7 = bf16_bits_to_f64(w.q)[2, 12:, 3]
    say("weights of bad pages and NaN keys")
    got = w.call(0.0)
    torch.cuda.synchronize()
    g = got.cpu().numpy()
    assert np.isnan(g[2, 0, 5])
    assert (g[2, 1, 6] == np.inf) if (q7 < 0).any() else g[2, 1, 6] == 0
    g[2, 0, 5] = g[2, 1, 6] = 0
    w.ks[2] = w.ks[2].copy()
    w.ks[2][5, 0] = w.ks[2][6, 1] = 0
    want, tol = key_weights(bf16_bits_to_f64(w.q), w.ks, w.lse.astype(np.float64), None, 0.0)
    want[2][0, 5] = want[2][1, 6] = 0
    for b, n in enumerate(w.lengths):
        assert np.max(np.abs(g[b, :, :n] - want[b]) / tol[b]) <= 1.0, b


def test_an_infinite_key_below_all_scores_weighs_nothing():
    """Ten heads in a tile of sixteen: rows of no head do not turn the key's weight into NaN."""
    w = Weights([40], 10, 1, page=32, seed=10)
    w.q[0, :, 9] = 0x3F80
    w.k.reshape(-1, 1, 128)[w.rows[0][3], 0, 9] = 0xFF80
    say("weights of a key at -inf")
    got = w.call(0.0)
    torch.cuda.synchronize()
    assert got[0, 0, 3].item() == 0.0 and torch.isfinite(got[0, 0, :40]).all()


def test_offsets_past_32_bits():
    """A pool of 6 GiB whose last pages hold the sequence."""
    page, H_KV = 256, 16
    pages = 6 * 2 ** 30 // (page * H_KV * 256)
    w = Weights([300], 16, H_KV, page, seed=11)
    pool = torch.zeros(pages, page, H_KV, 128, dtype=torch.bfloat16, device="cuda")
    own = w.table[0, :2].copy()
    place = np.array([pages - 1, pages - 3], dtype=np.int32)
    pool[torch.from_numpy(place.astype(np.int64)).cuda()] = to_dev(w.k)[torch.from_numpy(own.astype(np.int64)).cuda()]
    old = torch.from_numpy(w.old).cuda()
    say("weights in a pool of 6 GiB")
    table = torch.from_numpy(place[None].copy()).cuda()
    got = da.da_add_key_weights(to_dev(w.q), pool, table, w.seq_lens(), torch.from_numpy(w.lse).cuda(), old, w.L)
    torch.cuda.synchronize()
    w.check(got, 1.0, "6 GiB")


def test_a_captured_call_follows_lengths_and_runs_on_its_stream():
    w = Weights([300, 10, 0], 8, 2, page=32, seed=12, max_pages=20)
    q, k, table = to_dev(w.q), to_dev(w.k), torch.from_numpy(w.table).cuda()
    lens, lse, old = w.seq_lens(), torch.from_numpy(w.lse).cuda(), torch.from_numpy(w.old).cuda()
    out = torch.empty_like(old)
    graph = torch.cuda.CUDAGraph()
    say("weights captured")
    with torch.cuda.graph(graph):
        da.da_add_key_weights(q, k, table, lens, lse, old, w.L, 1.0, out)
    ks = w.ks
    for cut in ([300, 10, 0], [7, 10, 0], [129, 1, 0]):
        lens.copy_(torch.tensor(cut, dtype=torch.int32))
        out.copy_(old)
        graph.replay()
        torch.cuda.synchronize()
        w.lengths, w.ks = cut, [x[:n] for x, n in zip(ks, cut)]
        w.check(out, 1.0, f"replay {cut}")
    other = torch.cuda.Stream()
    out.copy_(old)
    torch.cuda.synchronize()
    a = da.da_add_key_weights(q, k, table, lens, lse, old, w.L, 1.0, out, stream=other)
    other.synchronize()
    w.check(a, 1.0, "other stream")
    b = da.da_add_key_weights(q, k, table, lens, lse, old, w.L, 1.0, old.clone())
    torch.cuda.synchronize()
    assert torch.equal(a, b)  # the same bits each time
