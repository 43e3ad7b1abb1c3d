"""The kernels that calls of the cache operators take for their size: rows with streaming hints, more tokens than waves
the chip holds, caches read past the last-level cache; and 4-bit steps bit for bit beside the bf16 ones."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import attend, kv4_unpack, visible_keys
from tests.cache_helpers import Batch, check_attention, normal_bits
from tests.gpu_helpers import say, to_dev
from tests.test_gpu_append import Step, bits, cache_rows, check_append, close, row_bytes
from tests.test_gpu_step import H_KV, H_Q, SLOTS_MAX, Server

pytestmark = pytest.mark.gpu

MIB = 1 << 20


def many_tokens():
    """More tokens than waves the chip holds (28 a CU)."""
    return 28 * torch.cuda.get_device_properties(0).multi_processor_count + 133


# tokens (None: more than the chip holds waves), heads, and the size in MiB moved (read and written) between the lines
# at which rows are written, and read too, with the streaming hint
SIZES = [(None, 5, 1, 0, 32), (2500, 21, 3, 32, 128), (None, 9, 1, 32, 128), (3500, 72, 4, 128, 1000),
         (None, 33, 3, 128, 1000)]


@pytest.mark.parametrize("N,heads,kv_heads,over,under", SIZES)
def test_appends_of_every_size(N, heads, kv_heads, over, under):
    N = N or many_tokens()
    assert over * MIB < N * (heads + 2 * kv_heads) * 512 <= under * MIB
    check_append(Step(N, heads, kv_heads, 32, seed=N, far=4000), f"N={N} {heads}/{kv_heads}", neighbours=heads % 2 == 0)


@pytest.mark.parametrize("N,heads,kv_heads,over,under", SIZES[1:2] + SIZES[3:])
def test_large_appends_in_place_and_without_q(N, heads, kv_heads, over, under):
    step = Step(N or many_tokens(), heads, kv_heads, 64, seed=heads, far=4000)
    (q, k, v, positions, slots), kw = step.device()
    q = q.contiguous()
    caches = [[to_dev(c) for c in step.cache] for _ in range(2)]
    say(f"append in place N={step.N} {heads}/{kv_heads}")
    got = da.da_append_kv(q, k, v, positions, slots, *caches[0], q_out=q, **kw)
    kw.pop("q_weight")
    assert da.da_append_kv(None, k, v, positions, slots, *caches[1], **kw) is None
    torch.cuda.synchronize()
    assert got is q
    close(q, step.exact("q"), "q in place")
    close(caches[0][0][slots.long()], step.exact("k"), "k")
    assert np.array_equal(bits(caches[0][1])[step.slots], step.v)
    for a, b in zip(*caches):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_four_bit_append_of_more_tokens_than_waves():
    N = many_tokens()
    rows = -(-(N + 40) // 64) * 64
    step = Step(N, 5, 1, 64, seed=8, rows=rows, far=4000)
    q, kb, vb = check_append(step, f"bf16 N={N}")
    cache = torch.zeros(rows // 64, 1, 2, 4352, dtype=torch.uint8, device="cuda")
    args, kw = step.device()
    say(f"append4 N={N}")
    q4 = da.da_append_kv4(*args, cache, **kw)
    torch.cuda.synchronize()
    assert torch.equal(q4.view(torch.int16), q.view(torch.int16))
    got = cache_rows(cache.cpu().numpy())
    assert np.array_equal(got[step.slots], np.concatenate([row_bytes(kb[step.slots]), row_bytes(vb[step.slots])], -1))
    assert not got[np.setdiff1d(np.arange(rows), step.slots)].any()


class Pool:
    """A 4-bit pool larger than what a launch reads without the streaming hint (64 MiB), and sequences in some of
    its pages."""

    def __init__(self, lengths, H_Q, H_KV, L, page, seed):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lengths, self.L, self.page, self.H_KV = lengths, L, page, H_KV
        tiles = page // 32
        self.num = 72 * MIB // (H_KV * tiles * 4352) + 1
        need = [-(-n // page) for n in lengths]
        assert sum(need) <= self.num
        self.cache = torch.randint(0, 256, (self.num, H_KV, tiles, 4352), dtype=torch.uint8, device="cuda", generator=g)
        self.cache[..., 4096:] = torch.randint(122, 128, (self.num, H_KV, tiles, 256), dtype=torch.uint8, device="cuda",
                                               generator=g)
        order = rng.permutation(self.num)
        self.table = rng.integers(0, self.num, (len(lengths), -(-L // page))).astype(np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.q = normal_bits(rng, (len(lengths), H_Q, 128))

    def streams(self, window, sinks):
        keys = da.da_window_keys(self.L, window, sinks) if window else self.L
        return min(len(self.lengths) * keys, self.num * self.page) * self.H_KV * 136 > 64 * MIB

    def check(self, window, sinks, splits, what):
        lens = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")
        lse = torch.empty(self.q.shape[:2], dtype=torch.float32, device="cuda")
        say(f"kv4 pool {what} W={window} S={sinks} splits={splits}")
        out = da.da_decode_attn_kv4(to_dev(self.q), self.cache, torch.from_numpy(self.table).cuda(), lens, self.L,
                                    window, sinks, lse_out=lse, num_splits=splits)
        torch.cuda.synchronize()
        check_attention(out, lse, self.reference(window, sinks), f"{what} W={window} splits={splits}")

    def reference(self, window, sinks):
        keys, values = [], []
        for b, n in enumerate(self.lengths):
            pages = torch.from_numpy(self.table[b, :-(-n // self.page)].astype(np.int64)).cuda()
            k, v = kv4_unpack(self.cache[pages].cpu().numpy()) if n else (np.zeros((0, self.H_KV, 128)),) * 2
            seen = visible_keys(n, window, sinks)
            keys.append(k[seen])
            values.append(v[seen])
        return attend(bf16_bits_to_f64(self.q), keys, values)


# one and two 16-column head tiles; a batch that is dealt and one sequence, whose chunks the host chooses
@pytest.mark.parametrize("heads,kv_heads,lengths,L", [
    (64, 8, [3000, 0, 41, 700, 2999, 64, 1, 1500], 9000), (64, 2, [5000, 33, 0, 900, 2, 2500, 320, 1], 36000),
    (64, 8, [9000], 70000), (64, 2, [7000], 270000)])
@pytest.mark.parametrize("windowed", [False, True])
def test_four_bit_caches_read_with_the_streaming_hint(heads, kv_heads, lengths, L, windowed):
    pool = Pool(lengths, heads, kv_heads, L, 256, seed=heads + len(lengths))
    window, sinks = (L - 100, 40) if windowed else (0, 0)
    for w in (window, 2000) if windowed else (0,):
        assert pool.streams(w, sinks) == (w != 2000)
        for splits in (0, 5):
            pool.check(w, sinks, splits, f"{heads}/{kv_heads} B={len(lengths)}")


@pytest.mark.parametrize("heads,kv_heads,B,window", [(64, 8, 64, 2500), (64, 2, 128, 2500), (16, 16, 40, 1100)])
@pytest.mark.parametrize("layout", ["packed", "paged"])
def test_windows_read_with_the_streaming_hint(heads, kv_heads, B, window, layout):
    """The windows of a batch hold more than the last-level cache (as far as the bound of the lengths says)."""
    rng = np.random.default_rng(B)
    lengths = [int(n) for n in rng.integers(0, 300, B)]
    lengths[3], lengths[B // 2], lengths[B - 1] = 4000, 2600, 3333
    batch = Batch(lengths, heads, kv_heads, layout, seed=B)
    keys = da.da_window_keys(batch.L, window, 70)
    for splits in (0, 3):
        assert da.da_make_plan(B, heads, kv_heads, keys, num_splits=splits).kv_nontemporal == 1
        lse = torch.empty(B, heads, dtype=torch.float32, device="cuda")
        say(f"window streamed {layout} {heads}/{kv_heads} splits={splits}")
        out = batch.call_window(da, window, 70, lse, num_splits=splits)
        torch.cuda.synchronize()
        check_attention(out, lse, batch.reference(window, 70), f"{layout} {heads}/{kv_heads} splits={splits}")


def test_four_bit_steps_hold_the_quantised_rows_of_the_bf16_steps():
    """Prompts, then decode steps as replays of a graph, over both caches: the 4-bit one holds, byte for byte, what the
    rows of the other quantise to, in every row of every step."""
    both = Server(False, seed=21), Server(True, seed=21)
    rng = both[0].rng

    def compare(buffers, before, what):
        slots = [b["slots"].cpu().numpy() for b in buffers]
        assert np.array_equal(*slots) and torch.equal(*(b["q"].view(torch.int16) for b in buffers)), what
        live = slots[0][slots[0] >= 0]
        rows, four = both[0].stored(), both[1].stored()
        want = np.concatenate([row_bytes(rows[0][live]), row_bytes(rows[1][live])], -1)
        assert live.size and np.array_equal(four[live], want), what
        rest = np.setdiff1d(np.arange(four.shape[0]), live)
        assert np.array_equal(four[rest], before[rest]), what

    def fill(buffers, new):
        x = to_dev(normal_bits(rng, (buffers[0]["x"].shape[0], H_Q + 2 * H_KV, 128), 2.0))
        for b in buffers:
            b["x"].copy_(x)
            b["new"].copy_(torch.tensor(new, dtype=torch.int32))

    for new in ([200, 1, 0, 333, 64, 95, 0, 0], [0, 40, 31, 7, 0, 300, 0, 0]):
        buffers = [s.buffers(sum(new) + 3) for s in both]
        fill(buffers, new)
        before = both[1].stored()
        say(f"both caches, prompts {new}")
        for s, b in zip(both, buffers):
            s.tables_and_rows(b)
        torch.cuda.synchronize()
        compare(buffers, before, f"prompts {new}")
    buffers = [s.buffers(SLOTS_MAX) for s in both]
    graphs = [torch.cuda.CUDAGraph() for _ in both]
    torch.cuda.synchronize()
    for s, b, graph in zip(both, buffers, graphs):
        with torch.cuda.graph(graph):
            s.tables_and_rows(b)
    for step in range(4):
        fill(buffers, [1, 1, 0, 1, 1, 1, 1, 0])
        before = both[1].stored()
        say(f"both caches, replay {step}")
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        compare(buffers, before, f"replay {step}")


def test_scale_bytes_of_every_bf16_value():
    """Appends write scale bytes from 2 to 252, and 255 where a block holds an infinity or a NaN, whatever the values."""
    x = np.arange(1 << 16).astype(np.uint16)
    rng = np.random.default_rng(22)
    x = np.concatenate([x, rng.permutation(x), np.sort(x & 0x7FFF), x & 0x80FF]).reshape(-1, 1, 128)
    cache = torch.zeros(x.shape[0] // 32, 1, 1, 4352, dtype=torch.uint8, device="cuda")
    say("scale bytes of every bf16 value")
    da.da_append_kv4(None, to_dev(x), to_dev(x), None, None, cache)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):  # signalling NaNs
        got, want = cache_rows(cache.cpu().numpy()), row_bytes(x)
    scales = got[..., 64:68]
    assert np.array_equal(scales, want[..., 64:]) and np.array_equal(got[..., 68:], got[..., :68])
    assert {2, 252, 255} <= set(np.unique(scales).tolist()) <= set(range(2, 253)) | {255}
    finite = (scales != 255).repeat(16, axis=-1)
    assert np.array_equal(got[..., :64][finite], want[..., :64][finite])
