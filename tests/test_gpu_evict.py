"""Eviction against the oracle: every output is a choice or a copy, so all are equal bit for bit."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle.cache import evict
from tests.cache_helpers import Batch
from tests.gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


class Evict(Batch):
    """Sequences with weights in which many rows are alike; `settled` rows have positions of earlier evictions."""

    def __init__(self, lengths, H_KV, page=64, seed=0, settled=0, spare=5, **kw):
        super().__init__(lengths, H_KV, H_KV, "paged", page, seed, **kw)
        rng = np.random.default_rng(seed + 1)
        B, stride = len(lengths), self.L + spare
        w = np.exp(2 * rng.standard_normal((B, H_KV, stride))).astype(np.float32)
        self.weights = np.where(w < 0.7, np.floor(w * 8) / 8, w).astype(np.float32)
        self.positions = np.full((B, H_KV, stride), -1, dtype=np.int32)
        self.totals = np.array(lengths, dtype=np.int32)
        for b, L in enumerate(lengths):
            if settled and L >= settled:
                self.totals[b] += 1000
                for h in range(H_KV):
                    self.positions[b, h, :settled] = rng.permutation(self.totals[b] - (L - settled))[:settled]
        self.free = rng.permutation(5000).astype(np.int32)
        self.taken = 3000

    def run(self, budget, sinks=0, recent=0, in_place=True, free=True, what="", L=None, call=None):
        ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        k, v, lens = to_dev(self.k), to_dev(self.v), self.seq_lens()
        w, p, f, taken = ints(self.weights), ints(self.positions), ints(self.free), ints(np.array([self.taken], np.int32))
        kw = dict(sinks=sinks, recent=recent)
        if free:
            kw.update(free_pages=f, taken=taken)
        if not in_place:
            kw.update(lens_out=torch.full_like(lens, 9), weights_out=torch.full_like(w, 9), positions_out=torch.full_like(p, 9))
            if free:
                kw["taken_out"] = torch.full_like(taken, 9)
        say(f"evict {what}")
        got = (call or da.da_evict_kv)(k, v, ints(self.table), lens, ints(self.totals), w, p, budget,
                                       self.L if L is None else L, **kw)
        torch.cuda.synchronize()
        if in_place:
            assert got[0] is lens and got[1] is w and got[2] is p
        else:
            assert torch.equal(lens, self.seq_lens()) and torch.equal(taken, ints(np.array([self.taken], np.int32)))
            assert np.array_equal(w.cpu().numpy().view(np.uint32), self.weights.view(np.uint32))
            assert np.array_equal(p.cpu().numpy(), self.positions)
        self.check(got, (k, v, f), budget, sinks, recent, in_place, free, what)
        return k, v, got

    def check(self, got, state, budget, sinks, recent, in_place, free, what):
        lens, w, p, moves, f, taken = evict(self.lengths, self.totals, self.weights, self.positions, self.table,
                                            self.page_of(), budget, sinks, recent, self.free, self.taken)
        same = lambda a, b: np.array_equal(a.view(np.uint32), b.view(np.uint32))  # noqa: E731
        assert np.array_equal(got[0].cpu().numpy(), lens), what
        gw, gp = got[1].cpu().numpy(), got[2].cpu().numpy()
        for b, n in enumerate(self.lengths):
            assert np.array_equal(gp[b, :, :n], p[b, :, :n]), f"{what}: positions of {b}"
            assert same(gw[b, :, :n].copy(), w[b, :, :n].copy()), f"{what}: weights of {b}"
            if in_place:
                assert same(gw[b, :, n:].copy(), self.weights[b, :, n:].copy())
                assert np.array_equal(gp[b, :, n:], self.positions[b, :, n:])
            else:
                assert (gw[b, :, n:] == 9).all() and (gp[b, :, n:] == 9).all()
        k, v, gf = state
        rows = self.k.shape[0] * self.k.shape[1]
        for x, was in ((k, self.k), (v, self.v)):
            y = was.reshape(rows, self.H_KV, 128).copy()
            src = was.reshape(rows, self.H_KV, 128)
            for b, h, d, s in moves:
                to, of = self.pool_row(b, d), self.pool_row(b, s)
                if to >= 0:
                    y[to, h] = src[of, h] if of >= 0 else 0
            assert np.array_equal(bits(x).reshape(y.shape), y), f"{what}: rows of the cache"
        if free:
            assert np.array_equal(gf.cpu().numpy(), f) and got[3].item() == taken, f"{what}: free pages"
        else:
            assert np.array_equal(gf.cpu().numpy(), self.free) and got[3] is None

    def page_of(self):
        return self.k.shape[1]

    def pool_row(self, b, r):
        page = int(self.table[b, r // self.page_of()])
        return page * self.page_of() + r % self.page_of() if 0 <= page < self.k.shape[0] else -1


@pytest.mark.parametrize("lengths,budget,sinks,recent", [
    ([1], 1, 0, 0), ([2], 1, 0, 0), ([2], 1, 0, 1), ([2], 1, 1, 0), ([33, 0, 32], 32, 4, 8), ([1000, 999, 1001], 999, 0, 1),
    ([1025, 64], 100, 100, 0), ([1025, 64], 100, 0, 100), ([1025, 700], 100, 50, 50), ([300, 500], 299, 7, 0),
    ([2000], 1999, 4, 33), ([2000], 1, 0, 0), ([0, 0], 5, 0, 0), ([1024, 2048, 1023], 1000, 3, 64),
])
@pytest.mark.parametrize("in_place", [True, False])
def test_lengths_around_the_budget(lengths, budget, sinks, recent, in_place):
    e = Evict(lengths, 2, 32, seed=budget)
    e.run(budget, sinks, recent, in_place, what=f"{lengths} to {budget}")


@pytest.mark.parametrize("page", [32, 96, 256])
@pytest.mark.parametrize("H_KV", [1, 3, 8])
@pytest.mark.parametrize("settled", [0, 200])
def test_pages_heads_and_history(page, H_KV, settled):
    e = Evict([513, 201, 200, 199, 0, 790], H_KV, page, seed=page + H_KV, settled=settled)
    e.run(200, 5, 40, what=f"page {page} heads {H_KV} settled {settled}")


@pytest.mark.parametrize("L", [4096, 4097, 8192, 8193, 16384, 16385, 40000])
@pytest.mark.parametrize("in_place", [True, False])
def test_every_kernel_variant(L, in_place):
    e = Evict([L, L // 2], 1, 64, seed=L, settled=100)
    e.run(1500, 10, 100, in_place, what=f"{L} rows")


def test_bounds_other_than_the_longest():
    e = Evict([700, 60, 200], 2, 32, seed=5, max_pages=2000, spare=63000)
    e.run(100, 2, 10, L=60000, what="L_K_max 60000")
    e = Evict([700, 60, 200], 2, 32, seed=6)
    w = e.weights.copy()
    k, v, got = None, None, None
    say("evict under a lower L_K_max")
    ints = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    k, v = to_dev(e.k), to_dev(e.v)
    totals = np.minimum(e.totals, 256).astype(np.int32)
    got = da.da_evict_kv(k, v, ints(e.table), e.seq_lens(), ints(totals), ints(w), ints(e.positions), 100, 256)
    torch.cuda.synchronize()
    e.lengths, e.totals = [256, 60, 200], totals
    e.check((*got[:3], None), (k, v, ints(e.free)), 100, 0, 0, True, False, "cut")


@pytest.mark.parametrize("budget", [100, 252, 300])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("captured", [False, True])
def test_sequences_past_the_bound_stay_as_they_are(budget, in_place, captured):
    """Lengths above L_K_max, below, at and above the budget: two launches, one, and nothing to evict within the
    bound.  Sequences 0 and 2 share the page of their sinks."""
    L, sinks, recent = 256, 32, 10
    e = Evict([700, 257, 256, 60, 200, 290], 2, 32, seed=34, settled=40)
    e.positions[0] = -1  # never evicted: row 0 is token 0
    e.totals[0] = 700
    e.positions[2, :, :32] = np.arange(32)
    e.positions[2, :, 32:40] = [33, 40, 50, 60, 70, 80, 90, 100]
    e.table[2, 0] = e.table[0, 0]
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    k, v, lens, w, p, f = to_dev(e.k), to_dev(e.v), e.seq_lens(), ints(e.weights), ints(e.positions), ints(e.free)
    taken, table, totals = ints(np.array([e.taken], np.int32)), ints(e.table), ints(e.totals)
    outs = {}
    if not in_place:
        outs = dict(lens_out=torch.full_like(lens, 9), weights_out=torch.full_like(w, 9),
                    positions_out=torch.full_like(p, 9), taken_out=torch.full_like(taken, 9))
    call = lambda: da.da_evict_kv(k, v, table, lens, totals, w, p, budget, L, sinks=sinks, recent=recent,  # noqa: E731
                                  free_pages=f, taken=taken, **outs)
    say(f"evict past the bound, budget {budget} in place {in_place} captured {captured}")
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        graph.replay()
    else:
        got = call()
    torch.cuda.synchronize()
    want, ww, wp, moves, wf, left = evict(e.lengths, e.totals, e.weights, e.positions, e.table, 32, budget, sinks, recent,
                                          e.free, e.taken, bound=L)
    assert want.tolist() == [n if n > L else min(n, budget) for n in e.lengths]
    assert np.array_equal(got[0].cpu().numpy(), want) and got[3].item() == left
    assert np.array_equal(f.cpu().numpy(), wf)
    gw, gp = got[1].cpu().numpy(), got[2].cpu().numpy()
    for b, n in enumerate(e.lengths):
        assert np.array_equal(gp[b, :, :n], wp[b, :, :n]), f"positions of {b}"
        assert np.array_equal(gw[b, :, :n], ww[b, :, :n]), f"weights of {b}"
        rest = (e.weights[b, :, n:], e.positions[b, :, n:]) if in_place else (9, 9)
        assert (gw[b, :, n:] == rest[0]).all() and (gp[b, :, n:] == rest[1]).all()
    rows = e.k.shape[0] * 32
    for x, was in ((k, e.k), (v, e.v)):
        src = was.reshape(rows, 2, 128)
        y = src.copy()
        for b, h, d, s in moves:
            assert e.lengths[b] <= L
            y[e.pool_row(b, d), h] = src[e.pool_row(b, s), h]
        assert np.array_equal(bits(x).reshape(y.shape), y), "rows of the cache"


@pytest.mark.parametrize("kind", ["zeros", "one", "signs", "infinite", "nan", "all nan", "tiny", "negative"])
def test_weights_that_tie_or_are_not_numbers(kind):
    e = Evict([700, 1200], 2, 32, seed=7)
    rng = np.random.default_rng(8)
    some = rng.random(e.weights.shape) < 0.5
    w = e.weights
    if kind == "zeros":
        w[...] = 0
    elif kind == "one":
        w[...] = 1.5
    elif kind == "signs":
        w[...] = np.where(some, np.float32(0.0), np.float32(-0.0))
    elif kind == "infinite":
        w[some] = np.inf
        w[rng.random(w.shape) < 0.2] = -np.inf
    elif kind == "nan":
        w[some] = np.nan
    elif kind == "all nan":
        w[...] = np.nan
    elif kind == "tiny":
        w[...] = np.float32(2.0 ** -149) * rng.integers(0, 5, w.shape).astype(np.float32)
    else:
        w[...] = -w
    e.run(300, 3, 20, what=kind)


@pytest.mark.parametrize("over", [1, 2, 4, 5, 6, 7, 63, 64, 65])
@pytest.mark.parametrize("kind", ["mixed", "alike", "nan", "late"])
def test_a_few_rows_past_the_budget(over, kind):
    """Rows found one after the other up to 5, moved by the first launch up to 64; sequences with fewer and without."""
    n = 700
    e = Evict([n + over, n + 1, n, n + (over + 1) // 2, 0, 5], 2, 32, seed=30 + over, settled=400)
    if kind == "alike":
        e.weights[...] = 0.25
    elif kind == "nan":
        e.weights[:, :, ::3] = np.nan
        e.weights[:, :, 1::5] = np.inf
    elif kind == "late":
        e.weights[:, :, n:] = -1
    e.run(n, 4, 0 if kind == "late" else 33, what=f"{over} past, {kind}")
    e.run(n, 0, 0, in_place=False, what=f"{over} past, {kind}, nothing protected")


@pytest.mark.parametrize("L", [300, 900, 5000, 32768, 32769, 40000])
def test_a_few_rows_in_every_kernel_variant(L):
    for over in (1, 5, 6, 64):
        Evict([L, L - 1], 2, 64, seed=over, settled=100).run(L - over, 10, 50, over % 2 == 0, what=f"{over} of {L} rows")


def test_many_sequences_in_one_launch():
    rng = np.random.default_rng(31)
    e = Evict([int(x) for x in rng.integers(90, 130, 1500)], 1, 32, seed=31)
    for taken in (4700, 3):
        e.taken = taken
        e.run(96, 4, 16, what="1500 sequences")
    e.run(1, 0, 1, what="a budget of one")


def test_a_few_pages_outside_the_pool():
    e = Evict([300, 299], 2, 32, seed=32)
    e.weights[:, :, :290] = 1
    e.weights[:, :, 40:44] = 0
    e.weights[:, :, 260:] = 2
    e.table[0, 1], e.table[1, 9] = -1, 10 ** 6  # a target, a source
    e.run(296, what="pages outside")


def test_a_free_list_with_few_pages_in_use_and_none():
    e = Evict([900, 400, 1000], 1, 32, seed=9)
    for taken in (0, 1, 5, 17, 5000):
        e.taken = taken
        e.run(100, what=f"{taken} pages in use")
    e.run(100, free=False, what="no free list")
    e = Evict([900, 30, 1000], 1, 32, seed=10)
    ints = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    say("evict with an empty free list")
    taken = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    da.da_evict_kv(to_dev(e.k), to_dev(e.v), ints(e.table), e.seq_lens(), ints(e.totals), ints(e.weights),
                   ints(e.positions), 100, e.L, free_pages=torch.empty(0, dtype=torch.int32, device="cuda"), taken=taken)
    torch.cuda.synchronize()
    assert taken.item() == 0


def test_many_sequences():
    rng = np.random.default_rng(11)
    e = Evict([int(x) for x in rng.integers(0, 300, 700)], 1, 32, seed=11)
    e.taken = 4700
    e.run(64, 4, 16, what="700 sequences")


def test_pages_outside_the_pool():
    e = Evict([300, 200], 2, 32, seed=12)
    e.table[0, 1], e.table[0, 8], e.table[1, 5] = -1, 10 ** 6, -(2 ** 31)
    e.run(96, what="pages outside")


def test_shared_pages_below_the_sinks_stay():
    e = Evict([400, 500], 2, 32, seed=13)
    e.table[1, :3] = e.table[0, :3]  # 96 shared keys
    e.run(200, 96, 20, what="shared pages")


def test_offsets_past_32_bits():
    page, H_KV = 256, 16
    pages = 6 * 2 ** 30 // (page * H_KV * 256)
    e = Evict([700], H_KV, page, seed=14)
    ids = torch.tensor([pages - 1, 2, pages - 2], device="cuda")
    pools = []
    own = torch.from_numpy(e.table[0, :3].astype(np.int64)).cuda()
    for x in (e.k, e.v):
        pool = torch.zeros(pages, page, H_KV, 128, dtype=torch.bfloat16, device="cuda")
        pool[ids] = to_dev(x)[own]
        pools.append(pool)

    def call(k, v, table, lens, *args, **kw):
        got = da.da_evict_kv(*pools, ids.int()[None].contiguous(), lens, *args, **kw)
        for x, pool in zip((k, v), pools):
            x[own] = pool[ids]
            pool[ids] = 0
            assert not pool.any()
        return got

    e.run(300, 4, 50, free=False, what="6 GiB pools", call=call)


def test_steps_in_a_row_keep_positions():
    """A key a step, evicted down to the budget each time: the rows are those of one choice by the sums of weights
    where later keys weigh more than all before, and the positions name the tokens."""
    budget, H_KV = 40, 2
    table = torch.arange(2, dtype=torch.int32, device="cuda")[None]
    k = torch.zeros(2, 32, H_KV, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    lens, totals = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    w = torch.zeros(1, H_KV, 64, device="cuda")
    p = torch.full((1, H_KV, 64), -1, dtype=torch.int32, device="cuda")
    score = np.random.default_rng(15).permutation(200)
    say("evict steps in a row")
    for t in range(200):
        row = int(lens)
        k.view(-1, H_KV, 128)[row] = float(t % 128)
        v.view(-1, H_KV, 128)[row] = float(t // 128)
        w[0, :, row] = float(score[t])
        lens += 1
        totals += 1
        da.da_evict_kv(k, v, table, lens, totals, w, p, budget, 64, sinks=3, recent=10)
        torch.cuda.synchronize()
        assert int(lens) == min(t + 1, budget)
        if t + 1 > budget:
            pos = p[0, 0, :budget].cpu().numpy()
            assert set(range(3)) <= set(pos) and set(range(t - 9, t + 1)) <= set(pos) and len(set(pos)) == budget
            for h in range(H_KV):
                tokens = k.view(-1, H_KV, 128)[:budget, h, 5].float() + 128 * v.view(-1, H_KV, 128)[:budget, h, 9].float()
                assert np.array_equal(tokens.cpu().numpy(), p[0, h, :budget].cpu().numpy())
    # a key stays once it is past the recent ones if it is among the best ever: the greedy choice keeps the best 27
    middle = sorted((t for t in range(3, 190)), key=lambda t: -score[t])[:27]
    assert set(middle) <= set(p[0, 0, :budget].cpu().numpy())


def test_captured_replays_follow_state_in_place():
    e = Evict([300, 120, 90], 2, 32, seed=16)
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    inputs = (to_dev(e.k), to_dev(e.v), e.seq_lens(), ints(e.weights), ints(e.positions), ints(e.free),
              ints(np.array([e.taken], np.int32)))
    k, v, lens, w, p, f, taken = (x.clone() for x in inputs)
    table, totals = ints(e.table), ints(e.totals)
    graph = torch.cuda.CUDAGraph()
    say("evict captured")
    with torch.cuda.graph(graph):
        got = da.da_evict_kv(k, v, table, lens, totals, w, p, 100, e.L, sinks=2, recent=9, free_pages=f, taken=taken)
    for i in range(3):
        for x, was in zip((k, v, lens, w, p, f, taken), inputs):
            x.copy_(was)
        graph.replay()
        torch.cuda.synchronize()
        e.check(got, (k, v, f), 100, 2, 9, True, True, f"replay {i}")
        da.da_evict_kv(k, v, table, lens, totals, w, p, 50, e.L)  # eager work between the replays
        torch.cuda.synchronize()


def test_a_callers_workspace_and_stream():
    e = Evict([300, 120], 2, 32, seed=17)
    need = da.da_evict_workspace_bytes(2, 2, e.L, 100)
    ws = torch.full((need,), 3, dtype=torch.uint8, device="cuda")
    ws[-(1 << 20):] = 0
    other = torch.cuda.Stream()
    torch.cuda.synchronize()

    def call(*args, **kw):
        torch.cuda.synchronize()
        got = da.da_evict_kv(*args, workspace=ws, stream=other, **kw)
        other.synchronize()
        return got

    for budget in (100, 295, 20, 299):  # two launches, one, two, one
        e.run(budget, 1, 2, what=f"own workspace, {budget}", call=call)
        assert not ws[-(1 << 20):].any()
    with pytest.raises(da.DecodeAttnError):
        e.run(100, what="short workspace", call=lambda *a, **kw: da.da_evict_kv(*a, workspace=ws[:need - 256], **kw))


def test_two_streams_at_once():
    """Each stream has its own counters; one launch a call, of many workgroups."""
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    streams, state = [torch.cuda.Stream() for _ in range(2)], []
    e = Evict([900 + b % 7 for b in range(60)], 8, 32, seed=33)
    for _ in range(6):
        state.append(dict(k=to_dev(e.k), v=to_dev(e.v), lens=e.seq_lens(), w=ints(e.weights), p=ints(e.positions),
                          free=ints(e.free), taken=ints(np.array([e.taken], np.int32))))
    table, totals = ints(e.table), ints(e.totals)
    torch.cuda.synchronize()
    say("evict on two streams")
    for i, s in enumerate(state):
        da.da_evict_kv(s["k"], s["v"], table, s["lens"], totals, s["w"], s["p"], 899, e.L, sinks=4, recent=40,
                       free_pages=s["free"], taken=s["taken"], stream=streams[i % 2])
    torch.cuda.synchronize()
    s = state[0]
    e.check((s["lens"], s["w"], s["p"], s["taken"]), (s["k"], s["v"], s["free"]), 899, 4, 40, True, True, "two streams")
    for other in state[1:]:
        assert all(torch.equal(other[name].view(torch.uint8), s[name].view(torch.uint8)) for name in s)
