"""Attention with a sliding window and sinks against the fp64 oracle."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from tests.cache_helpers import Batch, check_attention, new_lse
from tests.gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu

# (window, sinks): one key, below and at and past a tile, sinks in part of a tile, sinks that meet the window
WINDOWS = [(1, 0), (1, 1), (31, 0), (32, 32), (33, 4), (100, 65), (512, 4), (4000, 0), (7, 5000), (2 ** 31 - 1, 0)]


def run(batch, window, sinks, what, **kw):
    lse = new_lse(batch)
    say(f"window {what} W={window} S={sinks} {kw}")
    out = batch.call_window(da, window, sinks, lse, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("layout", ["dense", "packed", "paged"])
def test_windows(layout, window, sinks):
    lengths = [1000, 1000, 1000] if layout == "dense" else [0, 1, 31, 32, 33, 64, 500, 1000]
    batch = Batch(lengths, 8, 2, layout, seed=3)
    ref = batch.reference(window, sinks)
    for s in (0, 1, 5):
        check_attention(*run(batch, window, sinks, layout, num_splits=s), ref, f"{layout} W={window} S={sinks} s={s}")


@pytest.mark.parametrize("H_Q,H_KV", [(8, 1), (32, 1), (128, 2), (64, 8), (40, 8), (16, 16), (12, 4)])
@pytest.mark.parametrize("layout", ["packed", "paged"])
def test_heads(layout, H_Q, H_KV):
    batch = Batch([700, 2, 1333], H_Q, H_KV, layout, page=96, seed=H_Q)
    ref = batch.reference(300, 40)
    for s, pack in ((0, -1), (1, 1), (4, 0), (3, 2), (64, 1)):
        check_attention(*run(batch, 300, 40, f"{H_Q}/{H_KV}", num_splits=s, pack_gqa=pack), ref, f"{H_Q}/{H_KV} s={s}")


def test_every_offset_in_a_tile():
    """Lengths that put the window's first key and the last key on every row of a tile."""
    lengths = list(range(200, 264))
    batch = Batch(lengths, 4, 1, "paged", page=32, seed=9)
    for window, sinks in ((70, 3), (64, 33)):
        check_attention(*run(batch, window, sinks, "offsets"), batch.reference(window, sinks), f"offsets W={window}")


@pytest.mark.parametrize("layout", ["dense", "packed", "paged"])
@pytest.mark.parametrize("fill", [0x7FC0, 0xFF80, 0x7F7F])  # NaN, -inf, the largest finite value
def test_hidden_keys_do_not_reach_the_result(layout, fill):
    """The same bits whatever the invisible rows hold."""
    lengths = [900, 900] if layout == "dense" else [900, 41, 333]
    batch = Batch(lengths, 16, 2, layout, seed=5)
    for window, sinks in ((130, 10), (33, 0)):
        want, want_lse = run(batch, window, sinks, layout)
        k, v = batch.k.copy(), batch.v.copy()
        hidden = batch.hidden_rows(window, sinks)
        k.reshape(-1, 2, 128)[hidden] = fill
        v.reshape(-1, 2, 128)[hidden] = fill
        for s in (0, 1, 6):
            out, lse = run(batch, window, sinks, f"{layout} hidden {fill:#x}", kv=(to_dev(k), to_dev(v)), num_splits=s)
            check_attention(out, lse, batch.reference(window, sinks), f"hidden {fill:#x} s={s}")
        out, lse = run(batch, window, sinks, layout, kv=(to_dev(k), to_dev(v)))
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)


def test_stale_pages_between_sinks_and_window():
    """Table entries of pages without a visible key may name no page at all."""
    batch = Batch([4000, 2500], 8, 1, "paged", page=32, seed=6)
    ref = batch.reference(200, 20)
    for b, L in enumerate(batch.lengths):
        batch.table[b, 1:(L - 200) // 32] = 2 ** 30
    check_attention(*run(batch, 200, 20, "stale pages"), ref, "stale pages")


def test_a_window_over_everything_is_plain_attention():
    batch = Batch([600] * 2, 16, 4, "dense", seed=8)
    out, _ = run(batch, 600, 0, "whole")
    plain = da.da_decode_attn(to_dev(batch.q), to_dev(batch.k), to_dev(batch.v))
    check_attention(plain, None, batch.reference(0, 0), "plain")
    check_attention(out, None, batch.reference(0, 0), "whole")


def test_scale_long_context_and_loose_bound():
    batch = Batch([30000, 12345], 16, 2, "paged", page=256, seed=10)
    for window, sinks in ((4096, 128), (20, 0)):
        ref = batch.reference(window, sinks, 0.05)
        check_attention(*run(batch, window, sinks, "long", softmax_scale=0.05), ref, "long")
        batch2 = Batch([300, 12], 16, 2, "paged", page=256, seed=10, max_pages=200)
        check_attention(*run(batch2, window, sinks, "loose bound", L=50000), batch2.reference(window, sinks), "loose")


def test_captured_call_follows_the_lengths():
    batch = Batch([2000, 1500, 1800], 8, 2, "paged", page=64, seed=12)
    q, k, v = to_dev(batch.q), to_dev(batch.k), to_dev(batch.v)
    table, lens = torch.from_numpy(batch.table).cuda(), batch.seq_lens()
    out, lse = torch.empty_like(q), new_lse(batch)
    ws = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")
    call = lambda: da.da_decode_attn_window(q, k, v, 300, 8, None, table, lens, out, lse, L_K_max=2048,  # noqa: E731
                                            workspace=ws)
    call()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for lengths in ([2000, 1500, 1800], [1, 0, 700], [320, 299, 2000]):
        say(f"window replay {lengths}")
        batch.lengths = lengths
        batch.rows = [batch.table[b, np.arange(n) // 64].astype(np.int64) * 64 + np.arange(n) % 64
                      for b, n in enumerate(lengths)]
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out, lse, batch.reference(300, 8), f"replay {lengths}")
        eager = torch.empty_like(q)
        da.da_decode_attn_window(q, k, v, 300, 8, None, table, lens, eager, L_K_max=2048)
        assert torch.equal(eager.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("splits,heads", [(1, (8, 2)), (3, (8, 2)), (20, (64, 2)), (7, (128, 2)), (64, (8, 2))])
def test_a_visible_nan_reaches_its_heads(splits, heads):
    """A NaN in a visible key: the heads that read it give NaN, in whichever chunk it lies; others do not."""
    batch = Batch([3000, 3000], *heads, "packed", seed=13)
    batch.k[3000 + 2990, 1, 7] = 0x7FC0
    out, lse = run(batch, 2000, 64, f"visible NaN s={splits}", num_splits=splits)
    got, l = out.float().cpu().numpy(), lse.cpu().numpy()
    g = heads[0] // 2
    assert np.isnan(got[1, g:]).all() and np.isnan(l[1, g:]).all()
    assert np.isfinite(got[1, :g]).all() and np.isfinite(got[0]).all() and np.isfinite(l[0]).all()
