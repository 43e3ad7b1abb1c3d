"""The operators of a shared and bounded cache together, as a server's step makes the calls: tables, rows with
positions on three axes, attention of groups that share prefixes, the weights of their keys, eviction."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import attend, evict, extend_tables, key_weights, norm_rotate_axes
from tests.cache_helpers import check_attention, normal_bits
from tests.gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu

H_Q, H_KV, PAGE, BUDGET, SINKS, RECENT, L_MAX = 8, 2, 32, 128, 96, 16, 160
AXES = bytes([0] * 16 + [1] * 24 + [2] * 24)


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


class Server:
    """Five requests: three after one prompt of 96 tokens, two after another of 64; their pages off one free list."""

    def __init__(self, chunk_keys=0, seed=0):
        self.chunk_keys = chunk_keys
        rng = np.random.default_rng(seed)
        ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.groups, own = [(3, 96), (2, 64)], [10, 33, 1, 60, 25]
        self.cu, self.pre = ints([0, 3, 5]), ints([96, 64])
        self.B, self.pages = 5, 40
        order = rng.permutation(self.pages).astype(np.int32)
        table = np.full((5, L_MAX // PAGE), -1, np.int32)
        table[:3, :3], table[3:, :2] = order[:3], order[3:5]
        taken, lens = 5, []
        for b, n in enumerate(own):
            held = [96, 96, 96, 64, 64][b]
            lens.append(held + n)
            for j in range(held // PAGE, -(-lens[b] // PAGE)):
                table[b, j] = order[taken]
                taken += 1
        self.table, self.free, self.taken = ints(table), ints(order), ints([taken])
        self.lens, self.totals = ints(lens), ints(lens)
        self.k, self.v = (to_dev(normal_bits(rng, (self.pages, PAGE, H_KV, 128))) for _ in range(2))
        self.weights = torch.zeros(5, H_KV, L_MAX, device="cuda")
        self.positions = torch.full((5, H_KV, L_MAX), -1, dtype=torch.int32, device="cuda")
        self.one = ints([1] * 5)
        angle = np.arange(400)[:, None] * 10000.0 ** (-np.arange(64) / 64)
        self.rope = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], axis=1).astype(np.float32)).cuda()
        self.wq, self.wk = to_dev(normal_bits(rng, (128,))), to_dev(normal_bits(rng, (128,)))
        self.qkv = torch.empty(5, H_Q + 2 * H_KV, 128, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.empty(5, H_Q, device="cuda")

    STATE = ("table", "free", "taken", "lens", "totals", "k", "v", "weights", "positions", "lse")

    def state(self):
        return {name: getattr(self, name).clone() for name in self.STATE}

    def draw(self, step):
        rng = np.random.default_rng(1000 + step)
        self.qkv.copy_(to_dev(normal_bits(rng, (5, H_Q + 2 * H_KV, 128), 2.0)))

    def tables(self):
        _, _, _, self.slots, _ = da.da_extend_tables(self.lens, self.one, self.free, self.taken, self.table, PAGE,
                                                     self.pages, 5, lens_out=self.lens, taken_out=self.taken)
        # a patch of an image: the same time, its row and its column
        self.pos = torch.stack([self.totals // 16, self.totals % 16, self.totals % 7])
        self.totals += 1

    def append(self):
        self.q = da.da_append_kv_axes(self.qkv[:, :H_Q], self.qkv[:, H_Q:H_Q + H_KV], self.qkv[:, H_Q + H_KV:], self.pos,
                                      self.slots, self.k, self.v, rope=self.rope, axes=AXES, q_weight=self.wq,
                                      k_weight=self.wk)

    def attend(self):
        self.out = da.da_decode_attn_prefix(self.q, self.k, self.v, self.table, self.lens, self.cu, self.pre, L_MAX,
                                            lse_out=self.lse, chunk_keys=self.chunk_keys)

    def weigh(self):
        da.da_add_key_weights(self.q, self.k, self.table, self.lens, self.lse, self.weights, L_MAX, 0.9)

    def evict(self):
        da.da_evict_kv(self.k, self.v, self.table, self.lens, self.totals, self.weights, self.positions, BUDGET, L_MAX,
                       sinks=SINKS, recent=RECENT, free_pages=self.free, taken=self.taken)

    def step(self):
        self.tables()
        self.append()
        self.attend()
        self.weigh()
        self.evict()
        return self.out


def rows(table, b, n):
    j = np.arange(n)
    return table[b, j // PAGE].astype(np.int64) * PAGE + j % PAGE


# negative: the sharing launches, which so small a batch does not take by itself
@pytest.mark.parametrize("chunk_keys", [0, -1])
def test_each_call_of_a_step_against_the_oracle(chunk_keys):
    s = Server(chunk_keys)
    evicted = returned = 0
    for t in range(40):
        say(f"step {t}")
        s.draw(t)
        was = {n: x.cpu().numpy() for n, x in s.state().items() if n not in ("k", "v")}
        s.tables()
        torch.cuda.synchronize()
        table, lens, taken, _, slots, _ = extend_tables(was["lens"], [1] * 5, was["free"], was["taken"][0], was["table"],
                                                        PAGE, s.pages, 5)
        assert np.array_equal(s.table.cpu().numpy(), table) and np.array_equal(s.lens.cpu().numpy(), lens)
        assert np.array_equal(s.slots.cpu().numpy(), slots) and s.taken.item() == taken

        k0, v0 = bits(s.k).reshape(-1, H_KV, 128), bits(s.v).reshape(-1, H_KV, 128)
        s.append()
        torch.cuda.synchronize()
        k, v, x = (bits(y).reshape(-1, H_KV, 128) for y in (s.k, s.v, s.qkv))
        x = bits(s.qkv)
        rest = np.setdiff1d(np.arange(k.shape[0]), slots)
        assert np.array_equal(k[rest], k0[rest]) and np.array_equal(v[rest], v0[rest])
        assert np.array_equal(v[slots], x[:, H_Q + H_KV:])
        want, size = norm_rotate_axes(bf16_bits_to_f64(x[:, H_Q:H_Q + H_KV]), bf16_bits_to_f64(bits(s.wk)), 1e-6,
                                      s.rope.cpu().numpy(), s.pos.cpu().numpy(), AXES, False)
        # one rounding to bf16 and fewer than 2^7 of 32 bits of the magnitudes that make up the element
        assert np.all(np.abs(bf16_bits_to_f64(k[slots]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * size)

        s.attend()
        torch.cuda.synchronize()
        q = bf16_bits_to_f64(bits(s.q))
        kf, vf = bf16_bits_to_f64(k), bf16_bits_to_f64(v)
        ks = [kf[rows(table, b, lens[b])] for b in range(5)]
        check_attention(s.out, s.lse, attend(q, ks, [vf[rows(table, b, lens[b])] for b in range(5)], None), f"step {t}")

        old = s.weights.cpu().numpy()
        s.weigh()
        torch.cuda.synchronize()
        new, tol = key_weights(q, ks, s.lse.cpu().numpy().astype(np.float64),
                               [old[b, :, :lens[b]].astype(np.float64) for b in range(5)], float(np.float32(0.9)))
        got = s.weights.cpu().numpy()
        for b in range(5):
            assert np.all(np.abs(got[b, :, :lens[b]] - new[b]) <= tol[b])
            assert not got[b, :, lens[b]:].any()      # what eviction leaves for new keys

        free, at = s.free.cpu().numpy(), s.taken.item()
        p = s.positions.cpu().numpy()
        s.evict()
        torch.cuda.synchronize()
        lens2, w2, p2, moves, free2, taken2 = evict(lens, s.totals.cpu().numpy(), got, p, table, PAGE, BUDGET, SINKS,
                                                    RECENT, free, at)
        assert np.array_equal(s.lens.cpu().numpy(), lens2) and np.array_equal(s.weights.cpu().numpy(), w2)
        assert np.array_equal(s.positions.cpu().numpy(), p2)
        assert np.array_equal(s.free.cpu().numpy(), free2) and s.taken.item() == taken2
        k2, v2 = k.copy(), v.copy()
        for b, h, d, src in moves:
            to, of = rows(table, b, L_MAX)[d], rows(table, b, L_MAX)[src]
            k2[to, h], v2[to, h] = k[of, h], v[of, h]
        assert np.array_equal(bits(s.k).reshape(k2.shape), k2) and np.array_equal(bits(s.v).reshape(v2.shape), v2)
        evicted += int((lens - lens2).sum())
        returned += at - taken2
    assert evicted > 50 and returned > 50
    # the prompts' pages are what they were
    first = Server()
    for b, n in ((0, 96), (3, 64)):
        r = rows(first.table.cpu().numpy(), b, n)
        assert np.array_equal(bits(first.k).reshape(-1, H_KV, 128)[r], bits(s.k).reshape(-1, H_KV, 128)[r])


@pytest.mark.parametrize("chunk_keys", [0, -1])
def test_a_captured_step_gives_the_bits_of_the_eager_one(chunk_keys):
    eager, s = Server(chunk_keys), Server(chunk_keys)
    s.draw(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # before the capture, on a state of its own
        warm = Server(chunk_keys)
        warm.draw(0)
        warm.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    say("step captured")
    with torch.cuda.graph(graph):
        out = s.step()
    for t in range(30):
        eager.draw(t)
        want = eager.step()
        s.draw(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), t
        for name in Server.STATE:
            assert torch.equal(getattr(s, name), getattr(eager, name)), (t, name)
