"""Norms, rotation and the rows' way into the caches against the fp64 oracle."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import kv4_codes, kv4_pack, norm_rotate
from tests.cache_helpers import normal_bits
from tests.gpu_helpers import say, to_dev, to_f64
from workloads import f32_to_bf16_bits

pytestmark = pytest.mark.gpu

EPS = 1e-5


class Step:
    """One step's projections (q, k, v side by side in rows of `pad` spare elements more) and tables."""

    def __init__(self, N, H_Q, H_KV, rot=128, norm=True, seed=0, rows=None, far=5000, pad=0, magnitude=2.0):
        rng = np.random.default_rng(seed)
        self.N, self.H_Q, self.H_KV = N, H_Q, H_KV
        width = (H_Q + 2 * H_KV) * 128 + pad
        self.x = normal_bits(rng, (N, width), magnitude)
        heads = self.x[:, :width - pad].reshape(N, H_Q + 2 * H_KV, 128)
        self.q, self.k, self.v = heads[:, :H_Q], heads[:, H_Q:H_Q + H_KV], heads[:, H_Q + H_KV:]
        self.wq = normal_bits(rng, (128,)) if norm else None
        self.wk = normal_bits(rng, (128,)) if norm else None
        self.rope = self.positions = None
        if rot:
            angle = np.arange(far)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
            self.rope = np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32)
            self.positions = rng.integers(0, far, N).astype(np.int32)
        self.rows = N + 40 if rows is None else rows
        self.slots = rng.permutation(self.rows)[:N].astype(np.int32)
        self.cache = normal_bits(rng, (2, self.rows, H_KV, 128))

    def device(self):
        """q, k, v as slices of the projection's output, and the keyword arguments."""
        x = to_dev(self.x)
        heads = x[:, :(self.H_Q + 2 * self.H_KV) * 128].unflatten(1, (-1, 128))
        q = heads[:, :self.H_Q] if self.H_Q else None
        ints = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
        kw = {"eps": EPS, "rope": ints(self.rope),
              "q_weight": None if self.wq is None else to_dev(self.wq),
              "k_weight": None if self.wk is None else to_dev(self.wk)}
        return (q, heads[:, self.H_Q:self.H_Q + self.H_KV], heads[:, self.H_Q + self.H_KV:], ints(self.positions),
                ints(self.slots)), kw

    def exact(self, which, neighbours=False):
        x, w = (self.q, self.wq) if which == "q" else (self.k, self.wk)
        f = lambda b: None if b is None else bf16_bits_to_f64(b)  # noqa: E731
        return norm_rotate(f(x), f(w), EPS, self.rope, self.positions, neighbours)


def close(got, want, what):
    """Rounded to bf16 once (2^-8 of the value); the 32-bit steps before it (a mean of
    128 squares, root, reciprocal, two products of coefficients, two of the pair, one by
    the norm: fewer than 2^7 roundings of 2^-24 each) are off by at most 2^-17 of the
    magnitudes that make up the element, and again rounded with it."""
    y, size = want
    tol = 2.0 ** -8 * np.abs(y) + 2.0 ** -16 * size + 2.0 ** -133
    worst = np.max(np.abs(to_f64(got) - y) / tol, initial=0.0)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the tolerance"


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def check_append(step, what, neighbours=False):
    args, kw = step.device()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    say(f"append {what}")
    q = da.da_append_kv(*args, kc, vc, neighbours=neighbours, **kw)
    torch.cuda.synchronize()
    if step.H_Q:
        close(q, step.exact("q", neighbours), f"{what} q")
    kb, vb = bits(kc), bits(vc)
    close(kc[torch.from_numpy(step.slots.astype(np.int64)).cuda()], step.exact("k", neighbours), f"{what} k")
    assert np.array_equal(vb[step.slots], step.v)
    rest = np.setdiff1d(np.arange(step.rows), step.slots)  # rows without a token are as they were
    assert np.array_equal(kb[rest], step.cache[0][rest]) and np.array_equal(vb[rest], step.cache[1][rest])
    return q, kb, vb


@pytest.mark.parametrize("rot", [0, 16, 32, 64, 96, 112, 128])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotations_and_norms(rot, neighbours, norm):
    check_append(Step(13, 8, 2, rot, norm, seed=rot), f"rot={rot} neighbours={neighbours} norm={norm}", neighbours)


@pytest.mark.parametrize("H_Q,H_KV", [(1, 1), (8, 1), (5, 5), (64, 8), (40, 8), (128, 2), (6, 3), (0, 3)])
@pytest.mark.parametrize("N", [1, 2, 61, 300])
def test_heads_and_tokens(N, H_Q, H_KV):
    check_append(Step(N, H_Q, H_KV, 64, seed=N + H_Q, pad=8 * (N % 3)), f"N={N} {H_Q}/{H_KV}")


def test_many_tokens():
    """More tokens than waves the chip holds: a wave takes all heads of a token."""
    check_append(Step(5000, 4, 2, 128, seed=5), "N=5000")


def test_only_one_weight():
    step = Step(20, 4, 2, 128, seed=1)
    step.wq = None
    check_append(step, "k_weight only")
    step = Step(20, 4, 2, 128, seed=2)
    step.wk = None
    check_append(step, "q_weight only")


@pytest.mark.parametrize("magnitude", [1e-30, 1e-12, 1e12, 1e17])
def test_magnitudes(magnitude):
    check_append(Step(9, 4, 2, 64, seed=3, magnitude=magnitude), f"magnitude {magnitude}")


def test_slots_and_positions_outside():
    step = Step(12, 4, 2, 64, seed=4)
    step.slots[[0, 3, 5]] = [-1, step.rows, 2 ** 31 - 1]
    step.positions[[1, 2, 4]] = [-1, 5000, 2 ** 31 - 1]
    args, kw = step.device()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    say("append slots and positions outside")
    q = da.da_append_kv(*args, kc, vc, **kw)
    torch.cuda.synchronize()
    close(q, step.exact("q"), "q")
    ok = np.setdiff1d(np.arange(12), [0, 3, 5])
    k, size = step.exact("k")
    close(kc[torch.from_numpy(step.slots[ok].astype(np.int64)).cuda()], (k[ok], size[ok]), "k")
    rest = np.setdiff1d(np.arange(step.rows), step.slots[ok])
    assert np.array_equal(bits(kc)[rest], step.cache[0][rest]) and np.array_equal(bits(vc)[rest], step.cache[1][rest])


def test_no_slots_means_row_n_and_q_in_place():
    step = Step(17, 4, 2, 128, seed=6, rows=17)
    (q, k, v, positions, _), kw = step.device()
    q = q.contiguous()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    say("append in place")
    got = da.da_append_kv(q, k, v, positions, None, kc, vc, q_out=q, **kw)
    torch.cuda.synchronize()
    assert got is q
    close(q, step.exact("q"), "q in place")
    close(kc, step.exact("k"), "k rows")
    assert np.array_equal(bits(vc), step.v)


def test_infinities_stay_in_their_head():
    step = Step(3, 4, 1, 64, norm=False, seed=7)
    step.q[1, 2, 100] = 0x7F80   # a dim that does not turn
    step.q[1, 3, 3] = 0x7FC0     # NaN in one that does: its partner is 35
    args, kw = step.device()
    say("append infinities")
    q = to_f64(da.da_append_kv(*args, to_dev(step.cache[0]), to_dev(step.cache[1]), **kw))
    torch.cuda.synchronize()
    bad = ~np.isfinite(q)
    assert np.argwhere(bad).tolist() == [[1, 2, 100], [1, 3, 3], [1, 3, 35]]
    assert q[1, 2, 100] == np.inf


# ---------------------------------------------------------------- 4 bits


def cache_rows(cache):
    """[rows, H_KV, codes and scales of K and V] bytes, by row."""
    pages, H, blocks, _ = cache.shape
    t = cache.transpose(0, 2, 1, 3).reshape(-1, H, 4352)
    out = np.empty((t.shape[0], 32, H, 136), dtype=np.uint8)
    for r in range(32):
        for isv in (0, 1):
            out[:, r, :, 68 * isv:68 * isv + 64] = t[:, :, 2048 * isv + 64 * r:2048 * isv + 64 * r + 64]
            for g in range(4):
                out[:, r, :, 68 * isv + 64 + g] = t[:, :, 4096 + 4 * (4 * (r % 16) + g) + r // 16 + 2 * isv]
    return out.reshape(-1, H, 136)


def row_bytes(x):
    codes, scales = kv4_codes(x)
    return np.concatenate([codes[..., 0::2] | codes[..., 1::2] << 4, scales], axis=-1)


@pytest.mark.parametrize("page", [32, 96])
@pytest.mark.parametrize("N,H_Q,H_KV", [(1, 8, 1), (61, 8, 2), (200, 0, 3), (33, 64, 8), (5000, 4, 2)])
def test_four_bits_hold_what_the_bf16_cache_quantises_to(N, H_Q, H_KV, page):
    rows = -(-(N + 40) // page) * page
    step = Step(N, H_Q, H_KV, 128, seed=N, rows=rows)
    q, kb, vb = check_append(step, f"bf16 N={N}")
    before = kv4_pack(step.cache[0], step.cache[1], page)
    cache = torch.from_numpy(before).cuda()
    args, kw = step.device()
    say(f"append4 N={N} {H_Q}/{H_KV} page={page}")
    q4 = da.da_append_kv4(*args, cache, **kw)
    torch.cuda.synchronize()
    if H_Q:
        assert torch.equal(q4.view(torch.int16), q.view(torch.int16))
    got, old = cache_rows(cache.cpu().numpy()), cache_rows(before)
    want = np.concatenate([row_bytes(kb[step.slots]), row_bytes(vb[step.slots])], axis=-1)
    assert np.array_equal(got[step.slots], want)
    rest = np.setdiff1d(np.arange(rows), step.slots)
    assert np.array_equal(got[rest], old[rest])


def test_four_bit_rounding_at_every_border():
    """Ties, values next to them, the largest of a block around 6, 7 and 8 times a power of
    two, zeros of both signs, denormals, the largest finite values: bytes equal to a search over the codes."""
    vals = []
    for top in (4.0, 5.96875, 6.0, 6.96875, 7.0, 7.03125, 7.96875):
        for mid in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            for sign in (1, -1):
                block = np.zeros(32, dtype=np.float32)
                block[0] = top
                m = np.float32(mid * sign)
                block[1:4] = [m, m * np.float32(1 + 2 ** -7), m * np.float32(1 - 2 ** -8)]
                block[4] = -0.0
                block[5] = -top if sign < 0 else 0.5 * top
                vals.append(block)
    blocks = np.stack(vals)
    scaled = [blocks * np.float32(2.0 ** e) for e in (0, -3, 9, 100, -100)]
    x = f32_to_bf16_bits(np.concatenate(scaled)).reshape(-1)
    extra = np.zeros((5, 32), dtype=np.uint16)
    extra[0] = 0x0000
    extra[1, ::2] = 0x8000
    extra[2] = 0x0001 + np.arange(32)          # denormals
    extra[3] = 0x7F7F                          # the largest finite value
    extra[4] = 0x0080 + np.arange(32)          # the smallest normal ones
    x = np.concatenate([x, extra.reshape(-1)])
    x = np.concatenate([x, np.zeros(-x.size % (128 * 32), dtype=np.uint16)]).reshape(-1, 1, 128)
    k = to_dev(x)
    cache = torch.zeros(x.shape[0] // 32, 1, 1, 4352, dtype=torch.uint8, device="cuda")
    say("4-bit borders")
    da.da_append_kv4(None, k, k, None, None, cache)
    torch.cuda.synchronize()
    got = cache_rows(cache.cpu().numpy())
    want = row_bytes(x)
    assert np.array_equal(got[..., :68], want) and np.array_equal(got[..., 68:], want)


def test_four_bit_infinities_and_nan():
    x = normal_bits(np.random.default_rng(8), (32, 1, 128))
    x[3, 0, 40], x[7, 0, 127], x[9, 0, 0] = 0x7F80, 0xFFC0, 0xFF80
    cache = torch.zeros(1, 1, 1, 4352, dtype=torch.uint8, device="cuda")
    say("4-bit infinities")
    da.da_append_kv4(None, to_dev(x), to_dev(x), None, None, cache)
    k, v = da.da_read_kv4(cache)
    torch.cuda.synchronize()
    want = np.zeros((32, 128), dtype=bool)
    want[3, 32:64] = want[7, 96:] = want[9, :32] = True
    for t in (k, v):
        assert np.array_equal(np.isnan(to_f64(t))[:, 0], want)
