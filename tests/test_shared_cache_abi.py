"""The operators of a shared and bounded cache on the CPU: refusals (every call
below returns before any HIP call), host-side sizing, and their oracle."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle.cache import norm_rotate, norm_rotate_axes
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
