"""The binding without a GPU.  Whole numbers past a 32-bit int: what a C int cannot
hold is refused or counts as the largest int, and does not wrap around to some other number."""

from types import SimpleNamespace

import pytest
import torch

import paper_2604_00028_amd as da
from paper_2604_00028_amd import _binding as bnd

PAST = 2 ** 32  # wraps around to 0


def test_window_keys():
    assert da.da_window_keys(PAST, 5) == da.da_window_keys(2 ** 31 - 1, 5) == 64
    assert da.da_window_keys(PAST + 5, 100) == 160
    assert da.da_window_keys(-PAST + 5, 100) == -1
    assert da.da_window_keys(100, -PAST + 5) == da.da_window_keys(100, 5, -PAST + 5) == -1


def test_workspace_sizes():
    size = lambda *a, **k: da.da_kv4_workspace_bytes(*a, num_cus=256, **k)  # noqa: E731
    assert size(1, 64, 8, 2048, num_splits=4) > 0
    assert size(1, 64, 8, PAST + 2048, num_splits=4) == 0    # no such length
    assert size(1, 64, 8, 2048, num_splits=PAST + 4) == 0
    assert size(1, 64, 8, 2048, window=-PAST + 2000, num_splits=4) == 0
    assert size(1, 64, 8, 2048, sinks=-PAST, num_splits=4) == 0
    assert size(PAST + 1, 64, 8, 2048, num_splits=4) == size(1, 64, PAST + 8, 2048, num_splits=4) == 0
    # keys of a pool beyond 64 bits bound nothing
    assert size(1, 64, 8, 30000, 2 ** 64 + 5) == size(1, 64, 8, 30000, 2 ** 63 - 1)
    assert da.da_workspace_bytes(1, 64, 128, PAST + 4) == da.da_workspace_bytes(1, 64, 128, 2 ** 31 - 1)
    assert da.da_dealt_workspace_bytes(PAST + 1, 64, 8, 256) == 0


@pytest.mark.parametrize("kw", [dict(L_K_max=PAST + 100), dict(num_splits=PAST + 1), dict(pack_gqa=PAST),
                                dict(B=PAST + 1), dict(policy=PAST)])
def test_plans(kw):
    args = dict(B=1, H_Q=64, H_KV=8, L_K_max=512, num_cus=256)
    da.da_make_plan(**args)
    with pytest.raises(da.DecodeAttnError):
        da.da_make_plan(**{**args, **kw})


def test_schedules():
    da.da_make_schedule([100, 200], 64, 8, 1000, num_cus=256)
    for kw in (dict(L_K_max=PAST + 200), dict(pack_gqa=PAST), dict(cu_margin=PAST + 1)):
        with pytest.raises(da.DecodeAttnError):
            da.da_make_schedule([100, 200], 64, 8, **{"L_K_max": 1000, "num_cus": 256, **kw})
    made = lambda c: da.da_make_schedule([100, 200], 64, 8, 1000, num_cus=256, chunk_tiles=c)[1].tolist()  # noqa: E731
    assert made(-PAST + 1) == made(0) != made(1)  # no more than zero: chosen


def test_new_outputs_come_from_the_memory_of_the_calls_stream(monkeypatch):
    """A block of the current stream's memory may be waiting for work that is queued there."""
    entered = []

    class On:
        def __init__(self, handle):
            self.handle = handle

        def __enter__(self):
            entered.append(self.handle)

        def __exit__(self, *exc):
            entered.append(None)

    monkeypatch.setattr(bnd, "_stream", lambda dev, stream: 5 if stream is None else stream)
    monkeypatch.setattr(bnd, "_on", lambda dev, handle: handle)
    monkeypatch.setattr(bnd.torch.cuda, "stream", On)
    q = torch.ones(2, 3)
    for stream, want in ((None, []), (5, []), (7, [7, None]), (0, [0, None])):
        entered.clear()
        assert bnd._new_out(q, stream).shape == (2, 3) and entered == want


def test_a_workspace_is_checked_before_its_address_is_taken():
    """Memory the GPU cannot reach, or bytes that do not lie side by side, are no workspace."""
    dev = torch.device("cuda", 0)
    on = lambda device, contiguous=True: SimpleNamespace(  # noqa: E731
        device=device, get_device=lambda: -1 if device.index is None else device.index,
        is_contiguous=lambda: contiguous)
    bnd._usable(on(dev), dev)
    for ws in (torch.zeros(64, dtype=torch.uint8), on(torch.device("cuda", 1)), on(dev, contiguous=False)):
        with pytest.raises(ValueError):
            bnd._usable(ws, dev)


def test_four_bit_lengths_are_not_bounded_by_the_bytes_of_bf16_keys():
    size = lambda L, **k: da.da_kv4_workspace_bytes(1, 64, 8, L, num_splits=4, num_cus=256, **k)  # noqa: E731
    assert size(1 << 20) == size((1 << 20) - 1) == size(1 << 30) == da.da_workspace_bytes(1, 64, 128, 4)
    assert size((1 << 30) + 1) == 0

    def call(L):
        return bnd.load().da_decode_attn_kv4(*[0x100000] * 5, None, 1, 64, 8, 1 << 14, 1 << 17, 1, L, 128, 0.0, 0, 0, 4,
                                             0x100000, 1000, None)

    assert call((1 << 30) + 1) == bnd.DA_ERR_SHAPE
    # nothing refused before the workspace (too small), or the device (none here)
    assert call(1 << 20) == call(1 << 30) in (bnd.DA_ERR_WORKSPACE, bnd.DA_ERR_HIP, bnd.DA_ERR_UNSUPPORTED)
