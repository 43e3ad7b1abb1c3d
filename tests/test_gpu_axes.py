"""Appends with positions on several axes against the fp64 oracle."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import kv4_pack, norm_rotate_axes
from tests.gpu_helpers import say, to_dev
from tests.test_gpu_append import EPS, Step, bits, close

pytestmark = pytest.mark.gpu


def split(pairs, A, order):
    """The axis of each pair: axes taking turns, or one section after the other, of unequal sizes."""
    if order == "turns":
        return [i % A for i in range(pairs)]
    cuts = [pairs * (i + 1) * (i + 2) // (A * (A + 1)) for i in range(A)]
    return [next(a for a in range(A) if i < cuts[a]) for i in range(pairs)]


class AxesStep(Step):
    def __init__(self, N, H_Q, H_KV, rot, A, order="sections", **kw):
        super().__init__(N, H_Q, H_KV, rot, **kw)
        rng = np.random.default_rng(kw.get("seed", 0) + 100)
        self.axes = split(rot // 2, A, order)
        self.positions = rng.integers(0, self.rope.shape[0], (A, N)).astype(np.int32)

    def exact(self, which, neighbours=False):
        x, w = (self.q, self.wq) if which == "q" else (self.k, self.wk)
        f = lambda b: None if b is None else bf16_bits_to_f64(b)  # noqa: E731
        return norm_rotate_axes(f(x), f(w), EPS, self.rope, self.positions, self.axes, neighbours)


def check(step, what, neighbours=False):
    args, kw = step.device()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    say(f"append axes {what}")
    q = da.da_append_kv_axes(*args, kc, vc, neighbours=neighbours, axes=step.axes, **kw)
    torch.cuda.synchronize()
    if step.H_Q:
        close(q, step.exact("q", neighbours), f"{what} q")
    else:
        assert q is None
    close(kc[torch.from_numpy(step.slots.astype(np.int64)).cuda()], step.exact("k", neighbours), f"{what} k")
    kb, vb = bits(kc), bits(vc)
    assert np.array_equal(vb[step.slots], step.v)
    rest = np.setdiff1d(np.arange(step.rows), step.slots)
    assert np.array_equal(kb[rest], step.cache[0][rest]) and np.array_equal(vb[rest], step.cache[1][rest])
    return q, kb, vb


@pytest.mark.parametrize("rot", [16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("A", [1, 2, 3, 4])
@pytest.mark.parametrize("order", ["sections", "turns"])
def test_axes_of_pairs(rot, neighbours, A, order):
    check(AxesStep(7, 6, 2, rot, A, order, seed=rot + A), f"rot={rot} neighbours={neighbours} A={A} {order}", neighbours)


@pytest.mark.parametrize("H_Q,H_KV", [(8, 1), (64, 8), (128, 2), (6, 3), (0, 3)])
@pytest.mark.parametrize("N", [1, 2, 61, 300])
@pytest.mark.parametrize("norm", [False, True])
def test_heads_and_tokens(N, H_Q, H_KV, norm):
    check(AxesStep(N, H_Q, H_KV, 128, 3, seed=N + H_Q, pad=8 * (N % 3), norm=norm), f"N={N} {H_Q}/{H_KV}")


@pytest.mark.parametrize("H_Q,H_KV,N", [(4, 2, 5000), (64, 8, 2500)])
def test_many_tokens(H_Q, H_KV, N):
    """More tokens than waves the chip holds, and rows past the caches: the launches with streaming hints."""
    check(AxesStep(N, H_Q, H_KV, 128, 3, seed=5, far=200), f"N={N} {H_Q}/{H_KV}")


def test_positions_outside_the_table_and_slots_outside_the_cache():
    step = AxesStep(12, 4, 2, 64, 3, seed=4)
    step.positions[0, 1], step.positions[1, 2], step.positions[2, 3] = -1, step.rope.shape[0], 2 ** 31 - 1
    step.positions[:, 4] = -(2 ** 31)
    check(step, "positions outside")
    step.slots[[0, 3, 5]] = [-1, step.rows, 2 ** 31 - 1]
    args, kw = step.device()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    say("append axes slots outside")
    da.da_append_kv_axes(*args, kc, vc, axes=step.axes, **kw)
    torch.cuda.synchronize()
    rest = np.setdiff1d(np.arange(step.rows), step.slots)
    assert np.array_equal(bits(kc)[rest], step.cache[0][rest]) and np.array_equal(bits(vc)[rest], step.cache[1][rest])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("rot", [32, 128])
def test_text_tokens_get_what_one_axis_gives(four, neighbours, rot):
    """The same position on every axis: the bits of da_append_kv and da_append_kv4."""
    step = AxesStep(77, 8, 2, rot, 3, "turns", seed=9, rows=96)
    step.positions[1:] = step.positions[0]
    (q, k, v, positions, slots), kw = step.device()
    kw["neighbours"] = neighbours
    say("append axes of text tokens")
    if four:
        a, b = (torch.zeros(3, 2, 1, da.KV4_TILE_BYTES, dtype=torch.uint8, device="cuda") for _ in range(2))
        qa = da.da_append_kv4(q, k, v, positions[0].contiguous(), slots, a, **kw)
        qb = da.da_append_kv4_axes(q, k, v, positions, slots, b, axes=bytes(step.axes), **kw)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
    else:
        ka, va, kb, vb = (to_dev(step.cache[i % 2]) for i in range(4))
        qa = da.da_append_kv(q, k, v, positions[0].contiguous(), slots, ka, va, **kw)
        qb = da.da_append_kv_axes(q, k, v, positions, slots, kb, vb, axes=bytes(step.axes), **kw)
        torch.cuda.synchronize()
        assert np.array_equal(bits(ka), bits(kb)) and np.array_equal(bits(va), bits(vb))
    assert np.array_equal(bits(qa), bits(qb))


@pytest.mark.parametrize("N", [1, 45, 3001])
def test_four_bits_hold_the_rows_of_the_bf16_call(N):
    rows = -(-N // 32) * 32 + 32
    step = AxesStep(N, 8, 2, 128, 3, seed=N, rows=rows)
    (q, k, v, positions, slots), kw = step.device()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    cache = torch.from_numpy(kv4_pack(step.cache[0], step.cache[1], 32)).cuda()
    say(f"append axes into 4 bits, N={N}")
    qa = da.da_append_kv_axes(q, k, v, positions, slots, kc, vc, axes=step.axes, **kw)
    qb = da.da_append_kv4_axes(q, k, v, positions, slots, cache, axes=step.axes, **kw)
    torch.cuda.synchronize()
    assert np.array_equal(bits(qa), bits(qb))
    assert np.array_equal(cache.cpu().numpy(), kv4_pack(bits(kc), bits(vc), 32))


def test_a_captured_append_follows_positions_and_slots():
    step = AxesStep(33, 8, 2, 128, 3, seed=8)
    (q, k, v, positions, slots), kw = step.device()
    kc, vc = to_dev(step.cache[0]), to_dev(step.cache[1])
    q_out = torch.empty(33, 8, 128, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    say("append axes captured")
    with torch.cuda.graph(graph):
        da.da_append_kv_axes(q, k, v, positions, slots, kc, vc, axes=step.axes, q_out=q_out, **kw)
    for i in range(3):
        positions.copy_((positions + 17) % step.rope.shape[0])
        slots.copy_(slots.flip(0))
        step.positions, step.slots = positions.cpu().numpy(), slots.cpu().numpy()
        graph.replay()
        torch.cuda.synchronize()
        close(q_out, step.exact("q"), f"replay {i} q")
        close(kc[slots.long()], step.exact("k"), f"replay {i} k")
        assert np.array_equal(bits(vc)[step.slots], step.v)
