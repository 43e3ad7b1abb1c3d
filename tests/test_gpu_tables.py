"""Block tables and slots built on the GPU against plain loops: whole numbers, equal."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle.cache import extend_tables
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

NAMES = ("lens_out", "taken_out", "cu_new", "slots", "positions")


def state(lens, new, page, taken=3, pool=1.2, width=None, seed=0):
    """(lens, new, free, taken, table, num_pages): pages in random order, noise in unused entries."""
    rng = np.random.default_rng(seed)
    held = [-(-max(0, n) // page) for n in lens]
    need = sum(max(0, -(-(max(0, a) + max(0, b)) // page) - h) for a, b, h in zip(lens, new, held) if b < 10 ** 6)
    free = taken + int(need * pool)
    num = sum(held) + free + 1
    ids = rng.permutation(num)
    if width is None:
        width = max([-(-(max(0, a) + max(0, b)) // page) for a, b in zip(lens, new) if b < 10 ** 6] + [1]) + 1
    table = rng.integers(-5, num + 5, (len(lens), width)).astype(np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :min(n, width)] = ids[at:at + min(n, width)]
        at += n
    return np.array(lens, np.int32), np.array(new, np.int32), ids[at:at + free].astype(np.int32), taken, table, num


def check(lens, new, free, taken, table, num, page, max_tokens, what, in_place=False):
    want = extend_tables(lens, new, free, taken, table, page, num, max_tokens)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    dl, dn, df, dt, db = dev(lens), dev(new), dev(free), dev([taken]), dev(table)
    say(f"tables {what} in_place={in_place}")
    kw = {"lens_out": dl, "taken_out": dt} if in_place else {}
    got = da.da_extend_tables(dl, dn, df, dt, db, page, num, max_tokens, **kw)
    torch.cuda.synchronize()
    assert np.array_equal(db.cpu().numpy(), want[0]), f"{what}: table"
    for name, g, w in zip(NAMES, got, (want[1], [want[2]], want[3], want[4], want[5])):
        g = g.cpu().numpy()
        assert np.array_equal(g, w), f"{what}: {name} at {np.flatnonzero(g != np.asarray(w))[:5]}"
    if not in_place:
        assert np.array_equal(dl.cpu().numpy(), lens) and int(dt) == taken


@pytest.mark.parametrize("page", [1, 16, 32, 96, 4096])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 256, 257, 1000, 4096])
def test_decode_steps(B, page):
    rng = np.random.default_rng(B + page)
    lens = rng.integers(0, 300, B)
    s = state(lens, np.ones(B, int), page, seed=B)
    for in_place in (False, True):
        check(*s, page, B + 5, f"decode B={B} page={page}", in_place)


@pytest.mark.parametrize("pool", [0.0, 0.5, 0.97, 1.2])
def test_mixed_steps_with_a_short_list(pool):
    rng = np.random.default_rng(int(100 * pool))
    B = 300
    new = rng.choice([0, 0, 1, 1, 1, 40, 700], B)
    s = state(rng.integers(0, 5000, B), new, 64, pool=pool, seed=1)
    for in_place in (False, True):
        check(*s, 64, int(new.sum()), f"mixed pool={pool}", in_place)
        check(*s, 64, int(new.sum()) // 2, f"mixed pool={pool}, few rows", in_place)
        check(*s, 64, 0, f"mixed pool={pool}, no rows", in_place)


def test_a_long_prompt_among_idle_requests():
    lens = np.zeros(4096, int)
    new = np.zeros(4096, int)
    new[2048] = 70000
    s = state(lens, new, 16, seed=2)
    check(*s, 16, 70000 + 100, "long prompt", True)


def test_requests_that_do_not_fit_their_row():
    lens, new = [10, 64, 128, 0, 128, 100], [5, 64, 1, 129, 0, 28]
    check(*state(lens, new, 32, width=4, seed=3), 32, 400, "row full")


def test_lengths_out_of_range():
    lens, new = [-5, 7, 2 ** 31 - 1, 50, 0], [3, -2 ** 31, 1, 2 ** 31 - 1, 2]
    s = state([0, 7, 0, 50, 0], [3, 0, 0, 0, 2], 16, width=8, seed=4)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.from_numpy(s[4]).cuda()
    say("tables lengths out of range")
    lo, tk, cu, slots, pos = da.da_extend_tables(dev(lens), dev(new), torch.from_numpy(s[2]).cuda(), dev([s[3]]), table,
                                                 16, s[5], 64)
    torch.cuda.synchronize()
    assert lo.tolist() == [3, 7, 2 ** 30, 50, 0]                  # the last one's rows lie past max_tokens
    assert cu.tolist() == [0, 3, 3, 4, 2 ** 30, 2 ** 30]
    assert int(tk) == s[3] + 1 and slots[:3].tolist() == [int(s[2][s[3]]) * 16 + i for i in range(3)]
    assert slots[3:].tolist() == [-1] * 61 and pos[:3].tolist() == [0, 1, 2]


@pytest.mark.parametrize("taken", [-1, 10 ** 6, 2 ** 31 - 1])
def test_a_count_outside_the_list_grants_nothing(taken):
    lens, new, free, _, table, num = state([0, 5], [4, 1], 8, taken=0, seed=5)
    want = extend_tables(lens, new, free, max(taken, 0), table, 8, num, 8)
    dt = torch.tensor([taken], dtype=torch.int32, device="cuda")
    db = torch.from_numpy(table).cuda()
    say(f"tables taken={taken}")
    got = da.da_extend_tables(*(torch.from_numpy(a).cuda() for a in (lens, new, free)), dt, db, 8, num, 8)
    torch.cuda.synchronize()
    assert np.array_equal(db.cpu().numpy(), want[0]) and got[0].tolist() == want[1].tolist()
    assert got[3].tolist() == want[4].tolist() and int(got[1]) == want[2]


def test_steps_in_a_captured_graph():
    """A state advanced in place by replays: the tables after each as plain loops give them."""
    B, page = 70, 16
    rng = np.random.default_rng(6)
    lens, new, free, taken, table, num = state(rng.integers(0, 60, B), rng.integers(0, 9, B), page, pool=30.0, width=60, seed=6)
    dl, dn, df, dt, db = (torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
                          for a in (lens, new, free, [taken], table))
    outs = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (B + 1, 1500, 1500)]
    call = lambda: da.da_extend_tables(dl, dn, df, dt, db, page, num, 1500, dl, dt, *outs)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        say(f"tables replay {i}")
        table, lens, taken, cu, slots, positions = extend_tables(lens, new, free, taken, table, page, num, 1500)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(db.cpu().numpy(), table) and np.array_equal(dl.cpu().numpy(), lens) and int(dt) == taken
        for g, w in zip(outs, (cu, slots, positions)):
            assert np.array_equal(g.cpu().numpy(), w)


def test_pages_that_are_none():
    """Table entries and list entries outside the cache: no slot for the tokens they would hold."""
    lens, new, free, taken, table, num = state([10, 20, 0, 7], [30, 3, 40, 1], 16, seed=8)
    table[0, 0], table[1, 1], table[3, 0] = -1, num, 2 ** 31 - 1
    free[taken + 1], free[taken + 3] = -7, num + 5
    for in_place in (False, True):
        check(lens, new, free, taken, table, num, 16, 80, "bad pages", in_place)


def test_two_streams_at_once():
    """The same tables from two streams, with outputs of their own."""
    rng = np.random.default_rng(9)
    s = state(rng.integers(0, 900, 200), rng.integers(0, 50, 200), 32, seed=9)
    lens, new, free, taken, table, num = s
    want = extend_tables(lens, new, free, taken, table, 32, num, 6000)
    dev = [torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda() for a in (lens, new, free, [taken])]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    tabs = [torch.from_numpy(table).cuda() for _ in sides]
    torch.cuda.synchronize()
    say("tables on two streams")
    got = []
    for side, tab in zip(sides, tabs):
        with torch.cuda.stream(side):
            got.append(da.da_extend_tables(*dev, tab, 32, num, 6000))
    torch.cuda.synchronize()
    for out, tab in zip(got, tabs):
        assert np.array_equal(tab.cpu().numpy(), want[0])
        for g, w in zip(out, (want[1], [want[2]], want[3], want[4], want[5])):
            assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("B,extra", [(2, 0), (300, 0), (300, 3000)])
def test_a_list_too_short_for_one_request_serves_no_later_one(B, extra):
    """Pages go out in request order: after the first request that the list cannot serve none gets a page, also one
    that it could; requests that need none are extended before and after."""
    page = 16
    lens, new = np.full(B, 20), np.ones(B, int)          # a page and a part of one: room for the next key
    at = B // 2 - 1
    lens[at], new[at] = 0, 40 + extra                    # needs three pages (and more), the list holds one
    lens[B - 1], new[B - 1] = 0, 5                       # needs the one there is
    lens, new, free, taken, table, num = state(lens, new, page, taken=2, seed=10)
    free = free[:taken + 1]
    _, lens_out, taken_out, _, slots, _ = extend_tables(lens, new, free, taken, table, page, num, 4000)
    assert lens_out[at] == 0 and lens_out[B - 1] == 0 and taken_out == taken
    assert all(lens_out[b] == 21 for b in range(B - 1) if b != at)
    for in_place in (False, True):
        check(lens, new, free, taken, table, num, page, 4000, f"one page for {B} requests", in_place)
