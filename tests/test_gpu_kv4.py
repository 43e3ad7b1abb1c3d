"""Attention over the 4-bit cache against the fp64 oracle, and the cache read back."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import attend, kv4_pack, kv4_unpack
from tests.cache_helpers import Batch, check_attention, new_lse, normal_bits
from tests.gpu_helpers import say, to_dev, to_f64
from workloads import f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def run(batch, what, window=0, sinks=0, **kw):
    lse = new_lse(batch)
    say(f"kv4 {what} W={window} S={sinks} {[k for k in kw if k != 'cache']}")
    out = batch.call_kv4(da, window, sinks, lse, **kw)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("page", [32, 64, 96])
def test_read_back_is_exact(page):
    batch = Batch([200, 77], 6, 3, "kv4", page=page, seed=page)
    cache = torch.from_numpy(batch.cache).cuda()
    k, v = kv4_unpack(batch.cache)
    say(f"read all, page {page}")
    gk, gv = da.da_read_kv4(cache)
    torch.cuda.synchronize()
    assert np.array_equal(to_f64(gk), k) and np.array_equal(to_f64(gv), v)
    rows = k.shape[0]
    slots = [5, rows - 1, 0, -1, 5, rows, 31, 32, 2 ** 31 - 1]
    say(f"read rows, page {page}")
    gk, gv = da.da_read_kv4(cache, torch.tensor(slots, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for i, s in enumerate(slots):
        inside = 0 <= s < rows
        assert np.array_equal(to_f64(gk)[i], k[s] if inside else 0 * k[0]), s
        assert np.array_equal(to_f64(gv)[i], v[s] if inside else 0 * v[0]), s


def test_every_code_and_scale_reads_back():
    """All 256 code pairs under every scale byte from 2 to 252, and NaN under 255."""
    rng = np.random.default_rng(4)
    cache = rng.integers(0, 256, (4, 2, 2, 4352)).astype(np.uint8)
    scales = cache[..., 4096:].reshape(-1)
    scales[:] = 2 + np.arange(scales.size) % 251
    scales[::97] = 255
    cache[..., 4096:] = scales.reshape(4, 2, 2, 256)
    k, v = kv4_unpack(cache)
    say("all codes")
    gk, gv = da.da_read_kv4(torch.from_numpy(cache).cuda())
    torch.cuda.synchronize()
    for got, want in ((to_f64(gk), k), (to_f64(gv), v)):
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.nan_to_num(got, nan=1.0), np.nan_to_num(want, nan=1.0))


@pytest.mark.parametrize("H_Q,H_KV", [(8, 1), (32, 1), (128, 2), (64, 8), (40, 8), (16, 16), (12, 4), (1, 1)])
def test_heads_and_splits(H_Q, H_KV):
    batch = Batch([1, 700, 0, 1333, 32, 33], H_Q, H_KV, "kv4", page=96, seed=H_Q)
    ref = batch.reference(0, 0)
    for s in (0, 1, 2, 5, 17, 64):
        check_attention(*run(batch, f"{H_Q}/{H_KV} s={s}", num_splits=s), ref, f"{H_Q}/{H_KV} s={s}")


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 0), (32, 32), (33, 4), (100, 65), (7, 5000), (2 ** 31 - 1, 0)])
def test_windows(window, sinks):
    batch = Batch([0, 1, 31, 32, 33, 64, 500, 1000], 8, 2, "kv4", page=64, seed=3)
    ref = batch.reference(window, sinks)
    for s in (0, 1, 5):
        check_attention(*run(batch, f"s={s}", window, sinks, num_splits=s), ref, f"W={window} S={sinks} s={s}")


def test_every_length_to_three_tiles():
    lengths = list(range(97))
    batch = Batch(lengths, 4, 1, "kv4", page=32, seed=9)
    for s in (0, 1, 3):
        check_attention(*run(batch, "lengths", num_splits=s), batch.reference(0, 0), f"lengths s={s}")


@pytest.mark.parametrize("fill", [0x00, 0xFF])
def test_invisible_rows_do_not_reach_the_result(fill):
    """Rows past a sequence and outside the window: the same bits whatever codes and scales (NaN at 255) they hold."""
    batch = Batch([900, 41, 333], 16, 2, "kv4", page=64, seed=5)
    for window, sinks in ((0, 0), (130, 10), (33, 0)):
        want, want_lse = run(batch, "before", window, sinks)
        cache = batch.cache.copy()
        tiles = cache.transpose(0, 2, 1, 3)
        for row in np.flatnonzero(batch.hidden_rows(window, sinks)):
            r = row % 32
            t = tiles[row // 64, row % 64 // 32]
            for isv in (0, 1):
                t[:, 2048 * isv + 64 * r:2048 * isv + 64 * r + 64] = fill
                for g in range(4):
                    t[:, 4096 + 4 * (4 * (r % 16) + g) + r // 16 + 2 * isv] = fill
        cache = torch.from_numpy(np.ascontiguousarray(tiles.transpose(0, 2, 1, 3))).cuda()
        out, lse = run(batch, f"filled {fill:#x}", window, sinks, cache=cache)
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)
        check_attention(out, lse, batch.reference(window, sinks), f"filled {fill:#x}")


@pytest.mark.parametrize("H_Q,H_KV", [(8, 1), (128, 2), (6, 3)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 40)])
def test_mixed_batches_cut_by_their_lengths(H_Q, H_KV, window, sinks):
    """Batches whose lengths decide the chunks on the device: empty ones first, last and between, one long, all short."""
    for seed, lengths in enumerate([[0, 5000, 0, 33, 4097, 1, 0], [1, 31, 64], [3000] * 5, [0, 0], [9000, 9000],
                                    list(range(0, 140, 2)) + [6000]]):
        batch = Batch(lengths, H_Q, H_KV, "kv4", page=64, seed=seed, max_pages=150)
        out = run(batch, f"dealt {H_Q}/{H_KV} {lengths[:7]}", window, sinks, L=9000)
        check_attention(*out, batch.reference(window, sinks), f"dealt {lengths[:7]}")
    again = run(batch, "dealt again", window, sinks, L=9000)
    assert torch.equal(again[0].view(torch.int16), out[0].view(torch.int16)) and torch.equal(again[1], out[1])


@pytest.mark.parametrize("B", [1024, 1025])
def test_many_sequences_and_a_long_one(B):
    """On either side of the most sequences whose lengths decide the chunks."""
    lengths = [int(n) for n in np.random.default_rng(B).integers(0, 120, B)]
    lengths[B - 2] = 4000
    batch = Batch(lengths, 4, 1, "kv4", page=32, seed=19, max_pages=125)
    check_attention(*run(batch, f"B={B}"), batch.reference(0, 0), f"B={B}")


def test_a_nan_block_reaches_its_own_sequence_only():
    batch = Batch([100, 100], 4, 2, "kv4", page=32, seed=6)
    row = int(batch.rows[0][50])
    batch.cache[row // 32, 1, 0, 4096 + 4 * (4 * (row % 32 % 16) + 2) + row % 32 // 16 + 2] = 255  # V, head 1, dims 64-95
    out, lse = run(batch, "NaN block")
    got = to_f64(out)
    assert np.isnan(got[0, 2:, 64:96]).all() and np.isfinite(lse.cpu().numpy()).all()
    assert np.isfinite(got[1]).all() and np.isfinite(got[0, :2]).all()
    assert np.isfinite(got[0, 2:, :64]).all() and np.isfinite(got[0, 2:, 96:]).all()


def test_pages_outside_the_cache_read_as_zeros():
    batch = Batch([128], 4, 1, "kv4", page=32, seed=7)
    k, v = kv4_unpack(batch.cache)
    for bad in (-1, batch.cache.shape[0], 2 ** 31 - 1):
        table = batch.table.copy()
        batch.table[0, 1] = bad
        rows = batch.rows[0]
        kk, vv = k[rows].copy(), v[rows].copy()
        kk[32:64] = vv[32:64] = 0
        ref = attend(bf16_bits_to_f64(batch.q), [kk], [vv])
        check_attention(*run(batch, f"page {bad}"), ref, f"page {bad}")
        batch.table = table


def test_long_context_loose_bound_and_scale():
    batch = Batch([30001, 257, 12345], 16, 2, "kv4", page=256, seed=10, max_pages=200)
    ref = batch.reference(0, 0, 0.05)
    for s, L in ((0, 30001), (0, 51200), (64, 51200), (1, 51200)):
        check_attention(*run(batch, f"long s={s} bound {L}", softmax_scale=0.05, num_splits=s, L=L), ref, f"long s={s}")


def test_results_repeat_and_the_workspace_is_left_clean():
    batch = Batch([3000, 100, 1700, 2999], 64, 8, "kv4", page=64, seed=11)
    need = da.da_kv4_workspace_bytes(4, 64, 8, 3000, num_splits=16)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    first, _ = run(batch, "repeat", num_splits=16, workspace=ws)
    for _ in range(5):
        again, _ = run(batch, "repeat", num_splits=16, workspace=ws)
        assert torch.equal(again.view(torch.int16), first.view(torch.int16))
    assert int(ws[-(1 << 20):].sum()) == 0


def test_captured_call_follows_the_lengths():
    batch = Batch([2000, 1500, 1800], 8, 2, "kv4", page=64, seed=12)
    q, cache = to_dev(batch.q), torch.from_numpy(batch.cache).cuda()
    table, lens = torch.from_numpy(batch.table).cuda(), batch.seq_lens()
    out, lse = torch.empty_like(q), new_lse(batch)
    ws = torch.zeros(da.da_kv4_workspace_bytes(3, 8, 2, 2048), dtype=torch.uint8, device="cuda")
    call = lambda: da.da_decode_attn_kv4(q, cache, table, lens, 2048, 0, 0, out, lse, workspace=ws)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for lengths in ([2000, 1500, 1800], [1, 0, 700], [320, 299, 2000]):
        say(f"kv4 replay {lengths}")
        batch.lengths = lengths
        batch.rows = [batch.table[b, np.arange(n) // 64].astype(np.int64) * 64 + np.arange(n) % 64
                      for b, n in enumerate(lengths)]
        lens.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out, lse, batch.reference(0, 0), f"replay {lengths}")


def test_another_stream():
    batch = Batch([3000, 1234], 16, 2, "kv4", page=64, seed=13)
    want, _ = run(batch, "own stream")
    side = torch.cuda.Stream()
    say("kv4 side stream")
    q, cache = to_dev(batch.q), torch.from_numpy(batch.cache).cuda()
    table, lens = torch.from_numpy(batch.table).cuda(), batch.seq_lens()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    da.da_decode_attn_kv4(q, cache, table, lens, 3000, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("magnitude", [1e-30, 1e-3, 1e3, 1e25])
def test_query_magnitudes(magnitude):
    """The query's 8-bit parts over the whole range of exponents, and elements far below the largest one."""
    batch = Batch([300, 64], 8, 2, "kv4", page=64, seed=14)
    rng = np.random.default_rng(15)
    spread = 2.0 ** -rng.integers(0, 25, batch.q.shape).astype(np.float64)
    spread[1] = 1.0
    q = magnitude * spread * rng.standard_normal(batch.q.shape)
    batch.q = f32_to_bf16_bits(q.astype(np.float32))
    # scores around one whatever the magnitude
    check_attention(*run(batch, f"magnitude {magnitude}", softmax_scale=0.1 / magnitude),
                    batch.reference(0, 0, 0.1 / magnitude), f"magnitude {magnitude}")


@pytest.mark.parametrize("large", [1.0, 16.0, 256.0, 4096.0])
@pytest.mark.parametrize("length", [1, 20, 300])
def test_scores_hold_beside_a_large_query_element(length, large):
    """Log-sum-exps to 32 bits, also where one element of the query is far larger than the others.

    An element within 11 powers of two of the largest is exact, a smaller one off by
    2^-19 of the largest's power of two; three products of 16 partial sums each, cut
    at 2^-23 of sums below sum |q k|, and the cut of the codes' own sums, 2^-23 each;
    the exponent's scale, its logarithm and the sum of 300 probabilities 2^-20 more."""
    batch = Batch([length], 8, 2, "kv4", page=32, seed=20)
    q = bf16_bits_to_f64(batch.q) * np.where(np.arange(128) == 21, large, 1.0)
    batch.q = f32_to_bf16_bits(q.astype(np.float32))
    q = bf16_bits_to_f64(batch.q)[0]
    _, lse = run(batch, f"large {large} L={length}")
    want = batch.reference(0, 0)[1][0]
    keys = np.abs(kv4_unpack(batch.cache)[0][batch.rows[0]])
    top = 2.0 ** np.floor(np.log2(np.abs(q).max(1)))
    for h in range(8):
        lost = np.where(np.abs(q[h]) < 2.0 ** -11 * top[h], 2.0 ** -19 * top[h], 0.0)
        k = keys[:, h // 4]
        tol = (k @ (lost + 3 * 17 * 2.0 ** -23 * np.abs(q[h]))).max() / np.sqrt(128) + 2.0 ** -20 * (1 + abs(want[h]))
        err = abs(float(lse[0, h]) - want[h])
        assert err <= tol, f"head {h}: off by {err:.2e}, tolerance {tol:.2e}"


@pytest.mark.parametrize("splits", [1, 3])
def test_queries_that_are_not_finite(splits):
    batch = Batch([400], 8, 2, "kv4", page=64, seed=16)
    want, _ = run(batch, "finite", num_splits=splits)
    batch.q[0, 1, 5], batch.q[0, 6, 127] = 0x7F80, 0x7FC0
    out, lse = run(batch, "not finite", num_splits=splits)
    got = to_f64(out)[0]
    assert np.isnan(got[[1, 6]]).all() and np.isnan(lse.cpu().numpy()[0, [1, 6]]).all()
    keep = [0, 2, 3, 4, 5, 7]
    assert np.array_equal(got[keep], to_f64(want)[0][keep]) and np.isfinite(lse.cpu().numpy()[0, keep]).all()


@pytest.mark.parametrize("splits", [0, 1, 3, 20])
def test_a_nan_key_reaches_its_heads(splits):
    """A visible key with a NaN block: the heads that read it give NaN, in whichever chunk it lies; others do not."""
    batch = Batch([2000, 2000], 8, 2, "kv4", page=64, seed=18)
    row = int(batch.rows[1][1500])
    batch.cache[row // 64, 0, row % 64 // 32, 4096 + 4 * (4 * (row % 16) + 3) + row % 32 // 16] = 255  # K, head 0
    out, lse = run(batch, f"NaN key s={splits}", num_splits=splits)
    got, l = to_f64(out), lse.cpu().numpy()
    assert np.isnan(got[1, :4]).all() and np.isnan(l[1, :4]).all()
    assert np.isfinite(got[1, 4:]).all() and np.isfinite(got[0]).all() and np.isfinite(l[0]).all()


def test_far_rows_of_a_large_cache():
    """Rows past 4 GiB: written, read back and attended to, in the 4-bit and the bf16 cache."""
    H_KV, page = 8, 1024
    rng = np.random.default_rng(17)
    N = 100
    k, v, q = (normal_bits(rng, (N, H_KV, 128)), normal_bits(rng, (N, H_KV, 128)), normal_bits(rng, (1, 16, 128), 2.0))
    num = 4200                                       # 4.7 GB in 4 bits
    row0 = (num - 1) * page + 7 * 32 + 5
    slots = torch.arange(row0, row0 + N, dtype=torch.int32, device="cuda")
    cache = torch.empty(num, H_KV, page // 32, 4352, dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    say("far rows, 4 bits")
    da.da_append_kv4(None, to_dev(k), to_dev(v), None, slots, cache)
    gk, gv = da.da_read_kv4(cache, slots)
    torch.cuda.synchronize()
    kk, vv = kv4_unpack(kv4_pack(np.pad(k, ((0, 28), (0, 0), (0, 0))), np.pad(v, ((0, 28), (0, 0), (0, 0))), 128))
    assert np.array_equal(to_f64(gk), kk[:N]) and np.array_equal(to_f64(gv), vv[:N])
    # the sequence ends in the last page: its visible window is exactly the rows written
    table = torch.tensor([[num - 1]], dtype=torch.int32, device="cuda")
    L = 7 * 32 + 5 + N
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    lse = torch.empty(1, 16, dtype=torch.float32, device="cuda")
    out = da.da_decode_attn_kv4(to_dev(q), cache, table, lens, L, N, 0, lse_out=lse)
    torch.cuda.synchronize()
    check_attention(out, lse, attend(bf16_bits_to_f64(q), [kk[:N]], [vv[:N]]), "far rows, 4 bits")
    del cache
    num = 2100                                       # 4.4 GB of K in bf16
    row0 = (num - 1) * page + 7 * 32 + 5
    slots = torch.arange(row0, row0 + N, dtype=torch.int32, device="cuda")
    kc, vc = (torch.empty(num, page, H_KV, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert kc.numel() * 2 > 1 << 32
    say("far rows, bf16")
    da.da_append_kv(None, to_dev(k), to_dev(v), None, slots, kc, vc)
    out = da.da_decode_attn_window(to_dev(q), kc, vc, N, 0, None, table - table + num - 1, lens, L_K_max=L, lse_out=lse)
    torch.cuda.synchronize()
    assert torch.equal(kc.view(-1, H_KV, 128)[row0:row0 + N].view(torch.int16), to_dev(k).view(torch.int16))
    check_attention(out, lse, attend(bf16_bits_to_f64(q), [bf16_bits_to_f64(k)], [bf16_bits_to_f64(v)]), "far, bf16")
