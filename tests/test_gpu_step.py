"""The cache operators together, as a server runs them: tables from lengths,
norms, rotation and rows into the cache, attention, step after step, the decode
steps as replays of one captured graph."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import attend, extend_tables, kv4_unpack, norm_rotate, visible_keys
from paper_2604_00028_amd import _binding as bnd
from tests.cache_helpers import Batch, check_attention, new_lse, normal_bits
from tests.gpu_helpers import say, to_dev, to_f64
from tests.test_gpu_append import EPS, cache_rows, close, row_bytes

pytestmark = pytest.mark.gpu

H_Q, H_KV, PAGE, SLOTS_MAX, WIDTH = 16, 2, 32, 8, 40  # a batch of up to eight requests


class Server:
    """The state a server keeps on the device, and the same on the host."""

    def __init__(self, four, seed):
        rng = self.rng = np.random.default_rng(seed)
        self.four = four
        self.num_pages = 37  # a page more than the prompts take
        self.free = rng.permutation(self.num_pages).astype(np.int32)
        self.table = np.full((SLOTS_MAX, WIDTH), -1, np.int32)
        self.lens, self.taken = np.zeros(SLOTS_MAX, np.int32), 0
        self.wq, self.wk = normal_bits(rng, (128,)), normal_bits(rng, (128,))
        angle = np.arange(WIDTH * PAGE)[:, None] * 10000.0 ** (-np.arange(64) / 64)
        self.rope = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.d = dict(free=dev(self.free), table=dev(self.table), lens=dev(self.lens), rope=dev(self.rope),
                      taken=torch.zeros(1, dtype=torch.int32, device="cuda"), wq=to_dev(self.wq), wk=to_dev(self.wk))
        if four:
            self.cache = torch.zeros(self.num_pages, H_KV, PAGE // 32, 4352, dtype=torch.uint8, device="cuda")
        else:
            self.cache = torch.zeros(2, self.num_pages, PAGE, H_KV, 128, dtype=torch.bfloat16, device="cuda")

    def buffers(self, rows):
        e = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
        return dict(x=torch.zeros(rows, H_Q + 2 * H_KV, 128, dtype=torch.bfloat16, device="cuda"), new=e(SLOTS_MAX),
                    cu=e(SLOTS_MAX + 1), slots=e(rows), pos=e(rows),
                    q=torch.zeros(rows, H_Q, 128, dtype=torch.bfloat16, device="cuda"))

    def tables_and_rows(self, b):
        d, x = self.d, b["x"]
        da.da_extend_tables(d["lens"], b["new"], d["free"], d["taken"], d["table"], PAGE, self.num_pages, x.shape[0],
                            d["lens"], d["taken"], b["cu"], b["slots"], b["pos"])
        q, k, v = x[:, :H_Q], x[:, H_Q:H_Q + H_KV], x[:, H_Q + H_KV:]
        kw = dict(rope=d["rope"], q_weight=d["wq"], k_weight=d["wk"], eps=EPS, q_out=b["q"])
        if self.four:
            da.da_append_kv4(q, k, v, b["pos"], b["slots"], self.cache, **kw)
        else:
            da.da_append_kv(q, k, v, b["pos"], b["slots"], *self.cache, **kw)

    def attention(self, b, out, lse, ws, window, sinks):
        d, q = self.d, b["q"][:SLOTS_MAX]
        if self.four:
            da.da_decode_attn_kv4(q, self.cache, d["table"], d["lens"], WIDTH * PAGE, window, sinks, out, lse, workspace=ws)
        else:
            da.da_decode_attn_window(q, *self.cache, window, sinks, None, d["table"], d["lens"], out, lse,
                                     L_K_max=WIDTH * PAGE, workspace=ws)

    def advance(self, new, rows):
        """The host's step, and what the cache holds before it."""
        want = extend_tables(self.lens, new, self.free, self.taken, self.table, PAGE, self.num_pages, rows)
        return want, self.stored()

    def stored(self):
        if self.four:
            return cache_rows(self.cache.cpu().numpy())
        return self.cache.cpu().view(torch.int16).numpy().view(np.uint16).reshape(2, -1, H_KV, 128).copy()

    def check(self, want, before, x_bits, b, what):
        """Every table, row and cache byte of the device against the host's step."""
        self.table, self.lens, self.taken, cu, slots, pos = want
        got = [t.cpu().numpy() for t in (self.d["table"], self.d["lens"], b["cu"], b["slots"], b["pos"])]
        for g, w in zip(got, (self.table, self.lens, cu, slots, pos)):
            assert np.array_equal(g, w), what
        assert int(self.d["taken"]) == self.taken
        q, k, v = x_bits[:, :H_Q], x_bits[:, H_Q:H_Q + H_KV], x_bits[:, H_Q + H_KV:]
        f = bf16_bits_to_f64
        close(b["q"], norm_rotate(f(q), f(self.wq), EPS, self.rope, pos, False), f"{what}: q")
        after = self.stored()
        live = slots >= 0
        rest = np.setdiff1d(np.arange(self.num_pages * PAGE), slots[live])
        ky, size = norm_rotate(f(k), f(self.wk), EPS, self.rope, pos, False)
        if self.four:
            assert np.array_equal(after[rest], before[rest]), f"{what}: other rows"
            assert np.array_equal(after[slots[live]][..., 68:], row_bytes(v[live])), f"{what}: v"
            kv = kv4_unpack(self.cache.cpu().numpy())[0][slots[live]]
            # off the rotated key by a unit of the block's scale at most: half by rounding (a whole where 7 becomes
            # 6), and the key's own rounding moves it no further than the next code
            unit = 2.0 ** (after[slots[live]][..., 64:68].astype(float) - 127).repeat(32, -1)
            assert np.all(np.abs(kv - ky[live]) <= 2 * unit), f"{what}: k"
        else:
            assert np.array_equal(after[:, rest], before[:, rest]), f"{what}: other rows"
            rows = torch.from_numpy(slots[live].astype(np.int64)).cuda()
            close(self.cache[0].flatten(0, 1)[rows], (ky[live], size[live]), f"{what}: k")
            assert np.array_equal(after[1][slots[live]], v[live]), f"{what}: v"

    def check_attention(self, b, out, lse, window, sinks, what):
        """Against 64 bits over what the cache holds."""
        if self.four:
            k, v = kv4_unpack(self.cache.cpu().numpy())
        else:
            k, v = (bf16_bits_to_f64(x) for x in self.stored())
        rows = []
        for i in range(SLOTS_MAX):
            j = visible_keys(int(self.lens[i]), window, sinks)
            rows.append(self.table[i, j // PAGE].astype(np.int64) * PAGE + j % PAGE)
        q = to_f64(b["q"])[:SLOTS_MAX]
        check_attention(out, lse, attend(q, [k[r] for r in rows], [v[r] for r in rows]), what)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("window,sinks", [(50, 4), (400, 0)])
def test_prompts_then_captured_decode_steps(four, window, sinks):
    server = Server(four, seed=int(four) + window)
    rng = server.rng
    # prompts of six requests, in two steps; two places of the batch stay empty
    for step, new in enumerate(([200, 1, 0, 333, 64, 95, 0, 0], [0, 40, 31, 7, 0, 300, 0, 0])):
        rows = sum(new) + 5
        b = server.buffers(rows)
        x = normal_bits(rng, (rows, H_Q + 2 * H_KV, 128), 2.0)
        b["x"].copy_(to_dev(x))
        b["new"].copy_(torch.tensor(new, dtype=torch.int32))
        want, before = server.advance(new, rows)
        say(f"step: prompts {step} four={four}")
        server.tables_and_rows(b)
        torch.cuda.synchronize()
        server.check(want, before, x, b, f"prompts {step}")
    # decode: one token each, as one graph; one request gets the last page, another none when it needs one
    b = server.buffers(SLOTS_MAX)
    out = torch.empty(SLOTS_MAX, H_Q, 128, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(SLOTS_MAX, H_Q, dtype=torch.float32, device="cuda")
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    server.attention(b, out, lse, ws, window, sinks)  # loads the kernels
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        server.tables_and_rows(b)
        server.attention(b, out, lse, ws, window, sinks)
    for step in range(5):
        new = [1, 1, 1, 1, 1, 1, 0, 0] if step != 3 else [1, 1, 1, 1, 1, 1, 30, 0]  # (a new request: its rows do not fit)
        x = normal_bits(rng, (SLOTS_MAX, H_Q + 2 * H_KV, 128), 2.0)
        b["x"].copy_(to_dev(x))
        b["new"].copy_(torch.tensor(new, dtype=torch.int32))
        want, before = server.advance(new, SLOTS_MAX)
        torch.cuda.synchronize()
        say(f"step: decode replay {step} four={four}")
        graph.replay()
        torch.cuda.synchronize()
        server.check(want, before, x, b, f"decode {step}")
        server.check_attention(b, out, lse, window, sinks, f"decode {step}")
    assert server.taken == server.num_pages and int(server.lens[2]) == 32  # 31 keys, one more, no page for the next


def test_paged_attention_over_an_appended_cache():
    """The bf16 cache the step fills is the one da_decode_attn_paged reads."""
    server = Server(False, seed=9)
    new = [500, 3, 0, 64, 33, 1, 200, 31]
    b = server.buffers(sum(new))
    x = normal_bits(server.rng, (sum(new), H_Q + 2 * H_KV, 128), 2.0)
    b["x"].copy_(to_dev(x))
    b["new"].copy_(torch.tensor(new, dtype=torch.int32))
    want, before = server.advance(new, sum(new))
    say("step: paged")
    server.tables_and_rows(b)
    out = torch.empty(SLOTS_MAX, H_Q, 128, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(SLOTS_MAX, H_Q, dtype=torch.float32, device="cuda")
    da.da_decode_attn_paged(b["q"][:SLOTS_MAX], *server.cache, server.d["table"], server.d["lens"], 500, out, lse)
    torch.cuda.synchronize()
    server.check(want, before, x, b, "paged")
    server.check_attention(b, out, lse, 0, 0, "paged")


def test_calls_go_to_their_tensors_device(monkeypatch):
    """Where another device is current, the call is made again with the tensors' one current."""
    batch = Batch([300, 20], 8, 2, "kv4", seed=1)
    seen = []
    real = bnd._get_device

    def elsewhere():
        seen.append(1)
        return 7 if len(seen) == 1 else real()

    for call in (lambda: batch.call_kv4(da), lambda: da.da_read_kv4(torch.from_numpy(batch.cache).cuda())):
        say("step: another device current")
        want = call()
        seen.clear()
        monkeypatch.setattr(bnd, "_get_device", elsewhere)
        got = call()
        monkeypatch.setattr(bnd, "_get_device", real)
        assert len(seen) == 2
        for g, w in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
            assert torch.equal(g.view(torch.int16), w.view(torch.int16))


def test_binding_refuses_what_does_not_fit():
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    q, k = z(3, 8, 128), z(3, 2, 128)
    kc = z(64, 2, 128)
    say("refusals of the binding")
    bad = [
        lambda: da.da_append_kv(q, k, z(3, 1, 128), None, None, kc, kc),
        lambda: da.da_append_kv(z(2, 8, 128), k, k, None, None, kc, kc),
        lambda: da.da_append_kv(q.float(), k, k, None, None, kc, kc),
        lambda: da.da_append_kv(q.transpose(0, 1), k, k, None, None, kc, kc),
        lambda: da.da_append_kv(q, k, k, None, i(2), kc, kc),
        lambda: da.da_append_kv(q, k, k, None, i(3).long(), kc, kc),
        lambda: da.da_append_kv(q, k, k, None, None, kc, z(63, 2, 128)),
        lambda: da.da_append_kv(q, k, k, None, None, kc.transpose(0, 1), kc.transpose(0, 1)),
        lambda: da.da_append_kv(q, k, k, None, None, kc, kc, rope=z(9, 64, t=torch.float32)),
        lambda: da.da_append_kv(q, k, k, i(3), None, kc, kc, rope=z(9, 64)),
        lambda: da.da_append_kv(q, k, k, None, None, kc, kc, q_weight=z(64)),
        lambda: da.da_append_kv(None, k, k, None, None, kc, kc, q_out=q),
        lambda: da.da_append_kv4(q, k, k, None, None, z(2, 2, 1, 4000, t=torch.uint8)),
        lambda: da.da_append_kv4(q, k, k, None, None, z(2, 1, 1, 4352, t=torch.uint8)),
        lambda: da.da_append_kv(q, k, k, None, i(3).cpu(), kc, kc),
        lambda: da.da_decode_attn_kv4(q, z(2, 2, 1, 4352, t=torch.uint8), i(3, 1), i(3).cpu(), 32),
        lambda: da.da_decode_attn_kv4(q, z(2, 2, 1, 4352, t=torch.uint8), i(3, 1), i(3), 32, out=z(3, 8, 64)),
        lambda: da.da_decode_attn_kv4(q, z(2, 2, 1, 4352, t=torch.uint8), i(3, 1), i(3), 32, lse_out=z(3, 8)),
        lambda: da.da_decode_attn_window(q, z(2, 32, 2, 128), z(2, 32, 2, 128), 5, 0, None, i(3, 1), None, L_K_max=32),
        lambda: da.da_decode_attn_window(q, z(2, 32, 2, 128), z(2, 32, 2, 128), 5, 0, None, i(2, 1), i(3), L_K_max=32),
        lambda: da.da_extend_tables(i(3), i(2), i(5), i(1), i(3, 4), 16, 9, 3),
        lambda: da.da_extend_tables(i(3), i(3), i(5), i(2), i(3, 4), 16, 9, 3),
        lambda: da.da_extend_tables(i(3), i(3), i(5), i(1), i(4, 4), 16, 9, 3),
        lambda: da.da_extend_tables(i(3), i(3), i(5), i(1), i(3, 4), 16, 9, 3, slots=i(2)),
        lambda: da.da_extend_tables(i(3), i(3), i(5), i(1), i(3, 4).long(), 16, 9, 3),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", n)
    for call, code in [
            (lambda: da.da_append_kv(q[..., :64].contiguous(), k[..., :64].contiguous(), k[..., :64].contiguous(), None,
                                     None, kc[..., :64].contiguous(), kc[..., :64].contiguous()), bnd.DA_ERR_UNSUPPORTED),
            (lambda: da.da_append_kv(q, k, k, i(3), None, kc, kc, rope=z(9, 24, t=torch.float32)), bnd.DA_ERR_UNSUPPORTED),
            (lambda: da.da_decode_attn_window(q, z(3, 64, 2, 128), z(3, 64, 2, 128), 0), bnd.DA_ERR_ARG),
            (lambda: da.da_decode_attn_kv4(q, z(2, 2, 1, 4352, t=torch.uint8), i(3, 1), i(3), 33), bnd.DA_ERR_SHAPE),
            (lambda: da.da_extend_tables(i(5000), i(5000), i(5), i(1), i(5000, 4), 16, 9, 3), bnd.DA_ERR_SHAPE)]:
        with pytest.raises(da.DecodeAttnError) as e:
            call()
        assert e.value.code == code


def test_empty_calls():
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    say("empty calls")
    out = da.da_append_kv(z(0, 8, 128), z(0, 2, 128), z(0, 2, 128), None, None, z(4, 2, 128), z(4, 2, 128))
    assert out.shape == (0, 8, 128)
    k, v = da.da_read_kv4(z(0, 2, 1, 4352, t=torch.uint8))
    assert k.shape == v.shape == (0, 2, 128)
    lse = z(2, 8, t=torch.float32)
    out = da.da_decode_attn_kv4(z(2, 8, 128), z(0, 2, 1, 4352, t=torch.uint8), z(2, 1, t=torch.int32),
                                z(2, t=torch.int32), 0, lse_out=lse)
    torch.cuda.synchronize()
    assert not out.any() and torch.isneginf(lse).all()
    out = da.da_decode_attn_window(z(2, 8, 128), z(0, 32, 2, 128), z(0, 32, 2, 128), 9, 2, None, z(2, 1, t=torch.int32),
                                   z(2, t=torch.int32), L_K_max=0)
    torch.cuda.synchronize()
    assert not out.any()


@pytest.mark.parametrize("kind", ["kv4", "window"])
def test_graphs_without_a_workspace(kind):
    """Captured without a call before, replayed in the other order, beside each other and beside their stream's own calls."""
    batches = [Batch([1500], 8, 2, "kv4" if kind == "kv4" else "paged", page=64, seed=s) for s in (31, 32, 33)]
    calls, refs, outs = [], [], []
    for batch in batches:
        if kind == "kv4":
            q, cache = to_dev(batch.q), torch.from_numpy(batch.cache).cuda()
            table, lens = torch.from_numpy(batch.table).cuda(), batch.seq_lens()
            fn = lambda o, l, q=q, c=cache, t=table, n=lens: da.da_decode_attn_kv4(  # noqa: E731
                q, c, t, n, 1500, 0, 0, o, l, num_splits=9)
            refs.append(batch.reference(0, 0))
        else:
            q, k, v = to_dev(batch.q), to_dev(batch.k), to_dev(batch.v)
            table, lens = torch.from_numpy(batch.table).cuda(), batch.seq_lens()
            fn = lambda o, l, q=q, k=k, v=v, t=table, n=lens: da.da_decode_attn_window(  # noqa: E731
                q, k, v, 900, 100, None, t, n, o, l, L_K_max=1500, num_splits=9)
            refs.append(batch.reference(900, 100))
        calls.append(fn)
        outs.append((torch.empty_like(q), new_lse(batch)))
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph, fn, out in zip(graphs, calls, outs):
        say(f"{kind} capture")
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            fn(*out)
            fn(*out)
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), side]
    for turn in range(6):
        say(f"{kind} replays {turn}")
        for out, lse in outs:
            out.fill_(7.0)
            lse.fill_(7.0)
        torch.cuda.synchronize()
        for i in (1, 2, 0) if turn % 2 else (2, 0, 1):
            if turn == 0 and i == 0:
                continue  # the second graph's first replay comes before the first one's
            with torch.cuda.stream(streams[i]):
                for _ in range(4):
                    graphs[i].replay() if i < 2 else calls[2](*outs[2])
        torch.cuda.synchronize()
        for i in (1, 2) if turn == 0 else (0, 1, 2):
            check_attention(*outs[i], refs[i], f"{kind} turn {turn} call {i}")
    del graphs


def test_empty_slices_and_an_empty_rotation_table():
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    qkv, cache = z(6, 12, 128), z(4, 2, 128)
    say("empty slices")
    q, k, v = qkv[2:2, :8], qkv[2:2, 8:10], qkv[2:2, 10:]
    rope, none = z(9, 64, t=torch.float32), z(0, t=torch.int32)
    out = da.da_append_kv(q, k, v, none, none, cache, cache.clone(), rope=rope)
    torch.cuda.synchronize()
    assert out.shape == (0, 8, 128) and not cache.any()
    with pytest.raises(ValueError):  # not the same as no rotation
        da.da_append_kv(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], z(6, t=torch.int32), None, cache, cache, rope=rope[:0])


def test_bounds_past_an_int_are_refused():
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    q, table, lens = z(1, 8, 128), z(1, 1, t=torch.int32), z(1, t=torch.int32)
    say("bounds past an int")
    for call in (lambda: da.da_decode_attn_kv4(q, z(1, 2, 1, 4352, t=torch.uint8), table, lens, 2 ** 32),
                 lambda: da.da_decode_attn_window(q, z(1, 32, 2, 128), z(1, 32, 2, 128), 9, 0, None, table, lens,
                                                  L_K_max=2 ** 32)):
        with pytest.raises(bnd.DecodeAttnError) as e:
            call()
        assert e.value.code == bnd.DA_ERR_SHAPE
