"""The operators of a shared and bounded cache on the CPU: refusals (every call
below returns before any HIP call), host-side sizing, and their oracle."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle.cache import norm_rotate, norm_rotate_axes
from paper_2604_00028_amd._binding import _axis_bytes
from tests.test_cache_abi import ALIGN, ARG, FAKE, NULL, SHAPE, UNSUP, refused


def axes_call(lib, four=False, axes=bytes(64), num_axes=3, q=FAKE, k=FAKE, rope=FAKE, rot=128, positions=FAKE,
              slots=FAKE, qo=FAKE, kc=FAKE, vc=FAKE, N=4, H_Q=8, H_KV=1, d=128, page=64, pages=4, neighbours=0, qs=1024):
    head = (q, qs, k, 128, FAKE, 128, None, None, 1e-6, rope, 100, rot, neighbours, axes, num_axes, positions, slots, qo)
    if four:
        return lib.da_append_kv4_axes(*head, kc, page, pages, N, H_Q, H_KV, d, None)
    return lib.da_append_kv_axes(*head, kc, vc, 256, N, H_Q, H_KV, d, None)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(axes=None), NULL), (dict(rope=None), NULL), (dict(positions=None), NULL), (dict(k=None), NULL),
    (dict(num_axes=0), ARG), (dict(num_axes=5), ARG), (dict(num_axes=-1), ARG), (dict(axes=bytes([0] * 63 + [3])), ARG),
    (dict(axes=bytes([255] * 64)), ARG), (dict(axes=bytes([0, 1, 2, 1]), rot=8), UNSUP), (dict(rot=130), UNSUP),
    (dict(neighbours=2), ARG), (dict(positions=FAKE + 2), ALIGN), (dict(rope=FAKE + 4), ALIGN), (dict(kc=None), NULL),
    (dict(d=64), UNSUP), (dict(N=-1), SHAPE), (dict(qs=1023), ALIGN),
])
def test_axes_refusals(lib, four, kw, code):
    refused(axes_call(lib, four, **kw), code)


def test_axes_past_the_rotation_are_not_read(lib):
    # rope_dim 16: eight pairs; the ninth byte names no axis.  No tokens: nothing is launched.
    assert axes_call(lib, N=0, axes=bytes([0, 1, 2, 0, 1, 2, 0, 1, 99]), rot=16) not in (ARG, NULL, ALIGN, SHAPE)


def test_axes_python_refusals():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        da.da_append_kv_axes(bf(1, 8, 128), bf(1, 1, 128), bf(1, 1, 128), torch.zeros(3, 1, dtype=torch.int32), None,
                             bf(4, 1, 128), bf(4, 1, 128), rope=torch.zeros(4, 16), axes=[0] * 8)


@pytest.mark.parametrize("axes", [[0, 2, 1, 0, 2, 1, 0, 0], range(8), np.arange(8), np.arange(8, dtype=np.uint8),
                                  torch.arange(8), bytearray(range(8))])
def test_axes_are_taken_by_their_numbers(axes):
    assert _axis_bytes(axes, torch.zeros(4, 16)) == bytes(int(a) for a in axes)


@pytest.mark.parametrize("axes,error", [(16, TypeError), ([0.0] * 8, TypeError), ([256] * 8, ValueError), ([-1] * 8, ValueError)])
def test_axes_that_are_no_small_numbers(axes, error):
    with pytest.raises(error):
        _axis_bytes(axes, torch.zeros(4, 16))


@pytest.mark.parametrize("neighbours", [False, True])
def test_oracle_of_one_axis(neighbours):
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((5, 3, 128)), rng.standard_normal(128)
    rope = rng.standard_normal((9, 64)).astype(np.float32)
    pos = np.array([0, 8, 9, -1, 3])
    a = norm_rotate(x, w, 1e-5, rope, pos, neighbours)
    b = norm_rotate_axes(x, w, 1e-5, rope, np.stack([pos, 1 - pos]), [0] * 32, neighbours)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    c = norm_rotate_axes(x, w, 1e-5, rope, np.stack([1 - pos, pos]), [1] * 31 + [0], neighbours)[0]
    keep = [i for i in range(128) if i not in ((62, 63) if neighbours else (31, 63))]
    assert np.array_equal(a[0][..., keep], c[..., keep]) and not np.array_equal(a[0], c)


def weights_call(lib, q=FAKE, k=FAKE, table=FAKE, lens=FAKE, lse=FAKE, w=FAKE, out=FAKE, stride=2048, B=2, H_Q=8, H_KV=1,
                 page=64, max_pages=32, pages=64, L=2048, d=128, decay=1.0):
    return lib.da_add_key_weights(q, k, table, lens, lse, w, out, stride, B, H_Q, H_KV, page, max_pages, pages, L, d, 0.0,
                                  decay, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(lse=None), NULL),
    (dict(w=None), NULL), (dict(out=None), NULL), (dict(B=0), SHAPE), (dict(H_Q=9, H_KV=2), SHAPE), (dict(L=-1), SHAPE),
    (dict(max_pages=31), SHAPE), (dict(stride=2047), SHAPE), (dict(stride=-1), SHAPE), (dict(H_Q=1 << 17, B=1), SHAPE),
    (dict(d=64), UNSUP), (dict(page=48), UNSUP), (dict(decay=-0.5), ARG), (dict(decay=1.5), ARG),
    (dict(decay=float("nan")), ARG), (dict(q=FAKE + 8), ALIGN), (dict(k=FAKE + 2), ALIGN), (dict(lse=FAKE + 2), ALIGN),
    (dict(w=FAKE + 1), ALIGN), (dict(out=FAKE + 2), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(lens=FAKE + 1), ALIGN),
])
def test_weight_refusals(lib, kw, code):
    refused(weights_call(lib, **kw), code)


def evict_call(lib, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, totals=FAKE, w=FAKE, p=FAKE, wo=FAKE, po=FAKE, stride=2048,
               lo=FAKE, free=FAKE, taken=FAKE, to=FAKE, num_free=10, B=2, H_KV=2, page=64, max_pages=32, pages=64, L=2048,
               d=128, budget=100, sinks=4, recent=8, ws=FAKE, ws_bytes=1 << 30):
    return lib.da_evict_kv(k, v, table, lens, totals, w, p, wo, po, stride, lo, free, taken, to, num_free, B, H_KV, page,
                           max_pages, pages, L, d, budget, sinks, recent, ws, ws_bytes, None)


WS = -6


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL),
    (dict(totals=None), NULL), (dict(w=None), NULL), (dict(p=None), NULL), (dict(wo=None), NULL), (dict(po=None), NULL),
    (dict(lo=None), NULL), (dict(taken=None), NULL), (dict(to=None), NULL), (dict(free=None), NULL),
    (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(H_KV=0), SHAPE), (dict(L=-1), SHAPE), (dict(max_pages=31), SHAPE),
    (dict(stride=2047), SHAPE), (dict(num_free=-1), SHAPE), (dict(pages=1 << 25), SHAPE), (dict(d=64), UNSUP),
    (dict(page=16), UNSUP), (dict(budget=0), ARG), (dict(budget=-3), ARG), (dict(sinks=-1), ARG), (dict(recent=-1), ARG),
    (dict(sinks=60, recent=41), ARG), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), ARG), (dict(k=FAKE + 8), ALIGN),
    (dict(v=FAKE + 2), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(w=FAKE + 1), ALIGN), (dict(po=FAKE + 2), ALIGN),
    (dict(free=FAKE + 2), ALIGN), (dict(ws=FAKE + 8), ALIGN), (dict(ws=None), WS), (dict(ws_bytes=1 << 20), WS),
])
def test_evict_refusals(lib, kw, code):
    refused(evict_call(lib, **kw), code)


BIG = 1 << 40


def test_launches_of_2_32_threads_are_refused(lib):
    """What the checks before let through, on both sides of the line; the side below reaches the device check."""
    ok = (-7, UNSUP)
    for B, H, L in ((4096, 1024, 2048), (4096, 2048, 1000), (4096, 4096, 500)):
        kw = dict(L=L, budget=L - 1, sinks=0, recent=0, ws_bytes=BIG)
        refused(evict_call(lib, B=B, H_KV=H, **kw), SHAPE)
        assert da.da_evict_workspace_bytes(B, H, L, L - 1) == 0
        assert da.da_evict_workspace_bytes(B - 1, H, L, L - 1) > 0
        if not torch.cuda.is_available():
            assert evict_call(lib, B=B - 1, H_KV=H, **kw) in ok
    for B, H, L, mp in ((1 << 20, 16, 2048, 32), (1 << 17, 1, 1 << 18, 4096), ((1 << 23), 1, 2049, 33)):
        kw = dict(H_Q=H, H_KV=H, L=L, max_pages=mp, stride=L)
        refused(weights_call(lib, B=B, **kw), SHAPE)
        if not torch.cuda.is_available():
            assert weights_call(lib, B=B - 1, **kw) in ok


def test_evict_workspace_bytes():
    # a count and two lists of the rows that may move, a sequence and head; counters of other calls behind
    assert da.da_evict_workspace_bytes(1, 1, 100, 60) == 512 + (1 << 20)      # 4 (1 + 80) bytes
    assert da.da_evict_workspace_bytes(2, 8, 4097, 4096) == 256 + (1 << 20)
    assert da.da_evict_workspace_bytes(2, 8, 100, 200) == 256 + (1 << 20)     # nothing ever moves
    for bad in ((0, 1, 10, 5), (4097, 1, 10, 5), (1, 0, 10, 5), (1, 1, -1, 5), (1, 1, 10, 0)):
        assert da.da_evict_workspace_bytes(*bad) == 0


def prefix_call(lib, q=FAKE, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, cu=FAKE, pre=FAKE, out=FAKE, lse=None, B=4, G=2, H_Q=8,
                H_KV=1, page=64, max_pages=32, pages=64, L=2048, d=128, chunk=0, ws=FAKE, ws_bytes=1 << 40):
    return lib.da_decode_attn_prefix(q, k, v, table, lens, cu, pre, out, lse, B, G, H_Q, H_KV, page, max_pages, pages, L, d,
                                     0.0, chunk, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL),
    (dict(cu=None), NULL), (dict(pre=None), NULL), (dict(out=None), NULL), (dict(B=0), SHAPE), (dict(B=4097), SHAPE),
    (dict(G=5), SHAPE), (dict(G=-1), SHAPE), (dict(H_Q=9, H_KV=2), SHAPE), (dict(L=-1), SHAPE), (dict(max_pages=31), SHAPE),
    (dict(H_Q=1 << 17, H_KV=1 << 17, L=1, B=1, G=1), SHAPE), (dict(B=4096, H_Q=2048), SHAPE), (dict(d=64), UNSUP),
    (dict(page=48), UNSUP), (dict(q=FAKE + 8), ALIGN), (dict(k=FAKE + 2), ALIGN), (dict(out=FAKE + 4), ALIGN),
    (dict(cu=FAKE + 2), ALIGN), (dict(pre=FAKE + 1), ALIGN), (dict(lse=FAKE + 2), ALIGN), (dict(lens=FAKE + 2), ALIGN),
    (dict(ws=FAKE + 4), ALIGN),
])
def test_prefix_refusals(lib, kw, code):
    refused(prefix_call(lib, **kw), code)


def test_prefix_workspace_bytes():
    assert da.da_prefix_workspace_bytes(32, 1, 64, 8, 256) > 128 * 512 * 130 * 4 + (1 << 20)
    for bad in ((0, 0, 8, 1), (4097, 1, 8, 1), (4, 5, 8, 1), (4, -1, 8, 1), (4, 1, 9, 2), (4096, 1, 2048, 1)):
        assert da.da_prefix_workspace_bytes(*bad, 256) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would run")
def test_calls_that_pass_the_checks_reach_the_device_check(lib):
    for rc in (axes_call(lib), axes_call(lib, True), weights_call(lib), evict_call(lib), prefix_call(lib),
               prefix_call(lib, G=0, cu=None, pre=None),
               evict_call(lib, free=None, taken=None, to=None, num_free=0)):
        assert rc in (-7, UNSUP)


def test_python_refuses_tensors_of_the_cpu():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        da.da_add_key_weights(bf(1, 8, 128), bf(2, 32, 1, 128), ints(1, 2), ints(1), torch.zeros(1, 8), torch.zeros(1, 1, 64),
                              64)
    with pytest.raises(ValueError):
        da.da_evict_kv(bf(2, 32, 1, 128), bf(2, 32, 1, 128), ints(1, 2), ints(1), ints(1), torch.zeros(1, 1, 64),
                       ints(1, 1, 64), 32, 64)
