"""Attention of groups that share a prefix against the fp64 oracle."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import attend
from tests.cache_helpers import check_attention, normal_bits
from tests.gpu_helpers import say, to_dev, to_f64

pytestmark = pytest.mark.gpu


class Groups:
    """Groups of (sequences, prefix) with own lengths behind; pages that a prefix fills are shared, the one it ends in
    is copied; noise in every row and table entry that no sequence owns."""

    def __init__(self, groups, own, H_Q, H_KV, page=64, seed=0, max_pages=None, lens=None):
        rng = np.random.default_rng(seed)
        self.groups, self.H_Q, self.H_KV, self.page = groups, H_Q, H_KV, page
        sizes = [n for n, _ in groups]
        B = sum(sizes)
        of = np.repeat(np.arange(len(groups)), sizes)
        own = [own[b % len(own)] for b in range(B)]
        # own None: a sequence without keys
        self.lens = [0 if o is None else groups[of[b]][1] + o for b, o in enumerate(own)] if lens is None else lens
        self.cu = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        self.pre = np.array([p for _, p in groups], dtype=np.int32)
        self.L = max(self.lens)
        need = [-(-n // page) for n in self.lens]
        num = sum(need) + 8
        self.table = rng.integers(0, num, (B, max(max(need), 1) if max_pages is None else max_pages)).astype(np.int32)
        order = list(rng.permutation(num))
        self.k, self.v = (normal_bits(rng, (num, page, H_KV, 128)) for _ in range(2))
        first = {}
        for b in range(B):
            whole = min(int(self.pre[of[b]]), self.lens[b]) // page
            for j in range(need[b]):
                if j < whole and (of[b], j) in first:
                    self.table[b, j] = first[of[b], j]
                    continue
                self.table[b, j] = order.pop()
                if j < whole:
                    first[of[b], j] = self.table[b, j]
            rest = min(int(self.pre[of[b]]), self.lens[b]) % page
            if rest and need[b] > whole:
                part = self.table[b, whole]
                src = first.setdefault((of[b], whole, "part"), part)
                for x in (self.k, self.v):
                    x[part, :rest] = x[src, :rest]
                if rest > 0 and src != part and (of[b], whole) in first:
                    for x in (self.k, self.v):
                        x[part, :rest] = x[first[of[b], whole], :rest]
        # a shorter sequence's last page may be one that others share whole: its rows are copies of theirs
        for b in range(B):
            n = min(int(self.pre[of[b]]), self.lens[b])
            a = max((c for c in range(B) if of[c] == of[b]), key=lambda c: min(self.pre[of[c]], self.lens[c]))
            for j in range(-(-n // page)):
                rows = min(page, n - j * page)
                if self.table[b, j] != self.table[a, j]:
                    for x in (self.k, self.v):
                        x[self.table[b, j], :rows] = x[self.table[a, j], :rows]
        self.q = normal_bits(rng, (B, H_Q, 128), 2.0)

    def rows(self, b):
        j = np.arange(self.lens[b])
        return self.table[b, j // self.page].astype(np.int64) * self.page + j % self.page

    def reference(self, scale=None, lens=None):
        k, v = (bf16_bits_to_f64(x).reshape(-1, self.H_KV, 128) for x in (self.k, self.v))
        rows = [self.rows(b) if lens is None else self.rows(b)[:lens[b]] for b in range(len(self.lens))]
        return attend(bf16_bits_to_f64(self.q), [k[r] for r in rows], [v[r] for r in rows], scale)

    def call(self, lse=None, L=None, cu=None, pre=None, lens=None, table=None, kv=None, q=None, **kw):
        ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        k, v = kv or (to_dev(self.k), to_dev(self.v))
        return da.da_decode_attn_prefix(
            to_dev(self.q) if q is None else q, k, v, ints(self.table) if table is None else table,
            ints(np.array(self.lens, np.int32)) if lens is None else lens, ints(self.cu if cu is None else cu),
            ints(self.pre if pre is None else pre), self.L if L is None else L, lse_out=lse, **kw)

    def lse(self):
        return torch.full(self.q.shape[:2], 7.0, dtype=torch.float32, device="cuda")

    def check(self, what, **kw):
        """The sharing launches with chosen chunks (or those that kw asks for), and what the call takes by itself."""
        ref = self.reference()
        for chunk in [kw.pop("chunk_keys", -1), 0]:
            say(f"prefix {what} chunk_keys {chunk}")
            lse = self.lse()
            out = self.call(lse, chunk_keys=chunk, **kw)
            torch.cuda.synchronize()
            check_attention(out, lse, ref, f"{what}, chunk_keys {chunk}")
        return out


HEADS = [(8, 1), (64, 8), (32, 1), (16, 16), (40, 8), (128, 2), (64, 1), (6, 3), (12, 1)]


@pytest.mark.parametrize("H_Q,H_KV", HEADS)
@pytest.mark.parametrize("n", [1, 2, 3, 5, 9, 17, 33])
def test_heads_and_group_sizes(H_Q, H_KV, n):
    """Every kind of unit: up to 16, 32, 64 and 128 rows, and several of them."""
    Groups([(n, 200)], [1, 40, 0, 100], H_Q, H_KV, seed=n).check(f"{H_Q}/{H_KV} n={n}")


@pytest.mark.parametrize("prefix", [0, 1, 31, 32, 33, 64, 95, 96, 160, 1000, 2049])
@pytest.mark.parametrize("page", [32, 96, 256])
def test_prefix_lengths(prefix, page):
    Groups([(6, prefix)], [0, 1, 33, 70], 16, 2, page, seed=prefix + page).check(f"prefix {prefix} page {page}")


def test_groups_of_all_sizes_and_sequences_outside():
    groups = [(3, 0), (1, 500), (12, 700), (2, 65), (30, 40), (1, 0), (4, 1500)]
    g = Groups(groups, [5, None, 0, 300, 32, 1], 32, 4, 32, seed=1)
    a = g.check("many groups")
    # the last groups' sequences outside all groups: the same keys, nothing shared
    g.check("some outside", cu=g.cu[:4], pre=g.pre[:3])
    g.check("none", cu=np.zeros(1, np.int32), pre=np.zeros(0, np.int32))
    b = g.check("again")
    assert torch.equal(a, b)


def test_a_group_that_starts_late_and_empty_groups():
    g = Groups([(4, 0), (9, 300), (3, 0)], [7, 50], 16, 2, seed=2)
    cu = np.array([4, 4, 13, 13, 13, 13], np.int32)
    g.check("late start", cu=cu, pre=np.array([900, 300, 5, 2 ** 31 - 1, -7], np.int32))


@pytest.mark.parametrize("cu", [[0, 9, 4, 16], [-5, 9, 12, 30], [16, 9, 4, 0], [2 ** 31 - 1, -(2 ** 31), 3, 8]])
def test_groups_that_run_backwards_share_nothing(cu):
    g = Groups([(16, 0)], [70, 33, 0], 16, 2, seed=3)
    if cu == [-5, 9, 12, 30]:   # bounds are cut to the batch: groups of 9, 3 and 4 that share nothing
        pre = np.zeros(3, np.int32)
    else:
        pre = np.full(3, 64, np.int32)
    g.check(f"cu {cu}", cu=np.array(cu, np.int32), pre=pre)


def test_empty_and_short_sequences_within_a_group():
    g = Groups([(8, 512)], [None, 10, None, 0, 90, 33], 16, 2, seed=4)
    g.table[0, :] = g.table[2, :] = -1   # what has no keys is not read
    g.check("empty sequences")
    lens = [700, 512, 100, 0, 515, 64, 513, 600]
    Groups([(8, 512)], [0], 16, 2, 32, seed=5, lens=lens).check("shorter than the prefix")
    Groups([(8, 512)], [0], 16, 2, 32, seed=6, lens=[0] * 7 + [40]).check("one that has keys")
    g = Groups([(5, 512)], [0], 16, 2, 32, seed=7, lens=[0] * 5)
    for chunk in (0, -1):
        lse = g.lse()
        out = g.call(lse, L=0, chunk_keys=chunk)
        torch.cuda.synchronize()
        assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("chunk", [1, 32, 64, 100, 512, 10 ** 6, 2 ** 31 - 1])
def test_chosen_chunks(chunk):
    Groups([(3, 3001), (20, 1000), (2, 40)], [500, 1, 80], 32, 4, 32, seed=8).check(f"chunk {chunk}", chunk_keys=chunk)


def test_long_prefix_and_own_parts():
    """Page windows beyond 64 pages, 64 chunks of each kind, and a bound far above the lengths."""
    Groups([(4, 40001)], [9000, 1, 5000, 33], 8, 1, 32, seed=9).check("long, MQA")
    Groups([(2, 20000)], [9000, 1], 8, 1, 32, seed=10).check("long, whole", chunk_keys=10 ** 6)
    Groups([(20, 9000)], [3000, 100], 8, 1, 32, seed=11, max_pages=3000).check("long, many rows, one chunk",
                                                                              chunk_keys=10 ** 6, L=90000)


def test_many_sequences():
    rng = np.random.default_rng(12)
    sizes = [int(x) for x in rng.integers(1, 40, 40)]
    g = Groups([(n, int(rng.integers(0, 300))) for n in sizes], [int(x) for x in rng.integers(0, 200, 97)], 8, 1, 32,
               seed=12)
    g.check(f"{sum(sizes)} sequences")


@pytest.mark.parametrize("groups", [[(35, 64)], [(17, 28000), (18, 28000)]], ids=["four waves", "two waves"])
def test_own_keys_by_single_waves(groups):
    """Enough of the sequences' own keys for a wave each, without and with as much work over shared ones; the last of
    the places that eight chunks share stay empty."""
    Groups(groups, [1500, 1, 2900, 1700], 8, 8, 32, seed=25).check(f"own keys by waves, {groups}")


@pytest.mark.parametrize("H_Q,H_KV,own", [(64, 1, [4000, 1, 2900, 3300]), (128, 2, [3000, 700, 64]), (32, 1, [4000, 33]),
                                          (40, 8, [1200, 30])])
def test_single_waves_of_many_heads_and_sequences_that_write_their_output(H_Q, H_KV, own):
    """Enough own keys for a wave each (12288 tiles of units): 17 to 32 heads a unit, two units that read the same keys,
    and sequences outside all groups, of which those of one chunk write their output themselves."""
    prefix, readers = 64, H_KV * (2 if H_Q // H_KV > 32 else 1)
    per = sum(-(-own[i % len(own)] // 32) for i in range(12)) / 12
    B = -(-13500 // int(per * readers))
    g = Groups([(B - 12, prefix), (12, 0)], own, H_Q, H_KV, 32, seed=30)
    tiles = sum(-(-n // 32) - (prefix // 32 if b < B - 12 else 0) for b, n in enumerate(g.lens))
    assert tiles * readers >= 24 * 512 and g.L < 8192
    g.check(f"waves of {H_Q}/{H_KV} heads, {B} sequences", cu=g.cu[:2], pre=g.pre[:1])


def test_groups_whose_chunks_fill_the_cus():
    """Chunk lengths that are weighed against each other: few groups, and one more than are weighed."""
    for n in (1, 3, 16, 17):
        g = Groups([(9, 700 + 64 * i) for i in range(n)], [40, 3], 32, 4, 32, seed=26)
        g.check(f"{n} groups")


def test_most_requests():
    """4096 requests, each two a group."""
    g = Groups([(4096, 0)], [1, 40, 3, 0], 2, 2, 32, seed=13)
    g.check("4096 sequences", cu=np.arange(0, 4097, 2).astype(np.int32), pre=np.zeros(2048, np.int32))
    g.check("4096 groups", cu=np.arange(0, 4097).astype(np.int32), pre=np.full(4096, 5, np.int32))


def test_a_bound_below_the_lengths_cuts_them():
    g = Groups([(6, 300)], [200, 10], 16, 2, 32, seed=14)
    say("prefix under a lower L_K_max")
    for L, chunk in ((320, -1), (256, -1), (256, 0)):
        lse = g.lse()
        out = g.call(lse, L=L, chunk_keys=chunk)
        torch.cuda.synchronize()
        check_attention(out, lse, g.reference(lens=[min(n, L) for n in g.lens]), f"L_K_max {L}")


@pytest.mark.parametrize("rows", ["few", "many"])
def test_pages_outside_the_pool_read_as_zeros(rows):
    g = Groups([(2 if rows == "few" else 20, 320)], [40], 16, 2, 32, seed=15)
    g.table[:, 3] = [-1, 10 ** 6][rows == "many"]
    g.table[1, 10] = -(2 ** 31)
    k, v = (bf16_bits_to_f64(x).reshape(-1, 2, 128) for x in (g.k, g.v))
    ks, vs = [], []
    for b in range(len(g.lens)):
        at = g.table[b, np.arange(g.lens[b]) // 32]
        ok = (at >= 0) & (at < g.k.shape[0])
        r = np.where(ok, at.astype(np.int64) * 32 + np.arange(g.lens[b]) % 32, 0)
        ks.append(k[r] * ok[:, None, None])
        vs.append(v[r] * ok[:, None, None])
    say("prefix pages outside")
    for chunk in (-1, 0):
        lse = g.lse()
        out = g.call(lse, chunk_keys=chunk)
        torch.cuda.synchronize()
        check_attention(out, lse, attend(bf16_bits_to_f64(g.q), ks, vs, None), f"pages outside, chunk_keys {chunk}")


@pytest.mark.parametrize("n", [2, 6, 20])
@pytest.mark.parametrize("chunk", [-1, 0])
def test_values_that_are_not_finite_reach_their_rows_only(n, chunk):
    g = Groups([(n, 320), (2, 64)], [40], 16, 2, 32, seed=16)
    g.q[1, 3, 5] = 0x7FC0                                      # a query
    g.k.reshape(-1, 2, 128)[g.rows(n)[70], 1, 9] = 0x7FC0      # an own key of the second group
    g.v.reshape(-1, 2, 128)[g.rows(0)[330], 0, 4] = 0x7F80     # an own value of sequence 0, head 0
    # rows past the sequences and pages of no one hold NaN
    seen = np.zeros(g.k.shape[0] * 32, bool)
    for b in range(n + 2):
        seen[g.rows(b)] = True
    for x in (g.k, g.v):
        x.reshape(-1, 2, 128)[~seen] = 0x7FC0
    say(f"prefix NaN n={n} chunk_keys {chunk}")
    lse = g.lse()
    out = g.call(lse, chunk_keys=chunk)
    torch.cuda.synchronize()
    o, l = to_f64(out), lse.cpu().numpy()
    bad = np.zeros(o.shape[:2], bool)
    bad[1, 3] = True
    bad[n, 8:] = True
    assert np.array_equal(np.isnan(l), bad)
    inf = ~np.isfinite(o) & ~bad[..., None]
    assert np.isnan(o[bad]).all()
    assert np.argwhere(inf).tolist() == [[0, h, 4] for h in range(8)]
    g.v.reshape(-1, 2, 128)[g.rows(0)[330], 0, 4] = 0
    o[0, :8, 4] = 0
    ref_o, ref_l, size = attend(bf16_bits_to_f64(g.q), *[[np.nan_to_num(bf16_bits_to_f64(x).reshape(-1, 2, 128)[g.rows(b)])
                                for b in range(n + 2)] for x in (g.k, g.v)], None)
    keep = ~bad
    keep[0, :8] = False
    tol = (2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * np.abs(ref_o) * (1 + 2.0 ** -7)
    assert np.max((np.abs(o - ref_o) / tol)[keep]) <= 1.0


@pytest.mark.parametrize("n", [1, 2, 6, 9, 20])
@pytest.mark.parametrize("chunk", [-1, 0, 32])
def test_scores_of_minus_infinity_weigh_nothing(n, chunk):
    """Whole tiles of them: the first of the shared keys and of each wave's own, chunks of nothing else, and a sequence
    that has no other keys."""
    g = Groups([(n, 320), (3, 0)], [40, 200], 16, 2, 32, seed=29)
    g.q[:, :, 7] = 0x3F80  # 1
    seen, first = [], 4 * 32
    for b, rows in enumerate(g.rows(b) for b in range(n + 3)):
        L = len(rows)
        dead = np.zeros(L, bool)
        if b < n:
            dead[:first] = True                      # shared
            dead[320:352] = True                     # the first of its own
        elif b == n + 2:
            dead[:] = True
        else:
            dead[:min(first, L - 1)] = True          # the first tile of each of four waves
        g.k.reshape(-1, 2, 128)[rows[dead], :, 7] = 0xFF80
        seen.append(rows[~dead])
    k, v = (bf16_bits_to_f64(x).reshape(-1, 2, 128) for x in (g.k, g.v))
    ref = attend(bf16_bits_to_f64(g.q), [k[r] for r in seen], [v[r] for r in seen], None)
    say(f"prefix scores of -inf n={n} chunk_keys {chunk}")
    lse = g.lse()
    out = g.call(lse, chunk_keys=chunk)
    torch.cuda.synchronize()
    check_attention(out, lse, ref, f"scores of -inf n={n}, chunk_keys {chunk}")


@pytest.mark.parametrize("scale", [0.01, 1.0])
def test_scales(scale):
    g = Groups([(7, 300)], [33], 16, 2, 32, seed=17)
    lse = g.lse()
    say(f"prefix scale {scale}")
    out = g.call(lse, softmax_scale=scale, chunk_keys=-1)
    torch.cuda.synchronize()
    o, l, size = g.reference(float(np.float32(scale)))
    tol = (2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -8 * np.abs(o) * (1 + 2.0 ** -7)
    assert np.max(np.abs(to_f64(out) - o) / tol) <= 1.0
    # scores of up to 2^9 at scale 1: a few roundings of 2^-24 of their terms' magnitudes (2^11) and of the score
    assert np.max(np.abs(lse.cpu().numpy() - l)) <= 2.0 ** -13 * max(1.0, 11.3 * scale)


def test_offsets_past_32_bits():
    g = Groups([(3, 600)], [100, 1], 16, 16, 256, seed=18)
    pages = 6 * 2 ** 30 // (256 * 16 * 256)
    ids = pages - 1 - np.arange(g.k.shape[0])
    at = torch.from_numpy(ids).cuda()
    pools = []
    for x in (g.k, g.v):
        pool = torch.zeros(pages, 256, 16, 128, dtype=torch.bfloat16, device="cuda")
        pool[at] = to_dev(x)
        pools.append(pool)
    g.check("6 GiB pools", kv=tuple(pools), table=torch.from_numpy(ids[g.table].astype(np.int32)).cuda())


def test_same_as_the_paged_call_without_groups():
    """Both within their tolerance of the oracle; the log-sum-exp of both in 32 bits."""
    g = Groups([(5, 0)], [300, 64, 1], 64, 8, 64, seed=19)
    a = g.lse()
    b = g.lse()
    g.call(a, cu=np.zeros(1, np.int32), pre=np.zeros(0, np.int32), chunk_keys=-1)
    da.da_decode_attn_paged(to_dev(g.q), to_dev(g.k), to_dev(g.v), torch.from_numpy(g.table).cuda(),
                            torch.tensor(g.lens, dtype=torch.int32, device="cuda"), g.L, lse_out=b)
    torch.cuda.synchronize()
    assert torch.allclose(a, b, rtol=0, atol=2.0 ** -12)


def test_no_keys_at_all():
    Groups([(3, 0), (1, 0)], [None], 16, 2, 32, seed=27).check("no keys")
    g = Groups([(3, 64)], [5], 16, 2, 32, seed=28)
    for chunk in (-1, 0, 32):
        say(f"prefix without a bound {chunk}")
        lse = g.lse()
        out = g.call(lse, L=0, chunk_keys=chunk)
        torch.cuda.synchronize()
        assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("chunk", [-1, 0])
def test_captured_replays_follow_lengths_and_groups(chunk):
    g = Groups([(9, 640), (3, 100)], [100], 16, 2, 32, seed=20)
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    lens = ints(np.array(g.lens, np.int32))
    cu, pre = ints(g.cu), ints(g.pre)
    q, k, v, table, lse = to_dev(g.q), to_dev(g.k), to_dev(g.v), ints(g.table), g.lse()
    eager_out = da.da_decode_attn_prefix(q, k, v, table, lens, cu, pre, g.L, chunk_keys=chunk)
    graph = torch.cuda.CUDAGraph()
    say("prefix captured")
    with torch.cuda.graph(graph):
        out = da.da_decode_attn_prefix(q, k, v, table, lens, cu, pre, g.L, lse_out=lse, chunk_keys=chunk)
    full = list(g.lens)
    for i, (cut, groups) in enumerate([(0, g.pre), (60, g.pre), (99, np.array([200, 0])), (0, np.array([640, 64]))]):
        g.lens = [n - (cut if b % 2 else 0) for b, n in enumerate(full)]
        lens.copy_(torch.tensor(g.lens, dtype=torch.int32))
        pre.copy_(torch.from_numpy(groups.astype(np.int32)))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out, lse, g.reference(), f"replay {i}")
        if i == 0:
            assert torch.equal(out, eager_out)
        da.da_decode_attn_prefix(q, k, v, table, lens, cu, pre, g.L, chunk_keys=-1)  # eager work between the replays
        torch.cuda.synchronize()


def test_a_callers_workspace_and_stream():
    g = Groups([(9, 640)], [100], 16, 2, 32, seed=21)
    need = da.da_prefix_workspace_bytes(9, 1, 16, 2)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    ws[-(1 << 20):] = 0
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    say("prefix on another stream")
    for chunk in (-1, 0, -1):
        lse = g.lse()
        torch.cuda.synchronize()
        out = g.call(lse, workspace=ws, stream=other, chunk_keys=chunk)
        torch.cuda.synchronize()
        check_attention(out, lse, g.reference(), "own workspace")
        assert not ws[-(1 << 20):].any()
    with pytest.raises(da.DecodeAttnError):
        g.call(workspace=ws[:need - 256])
    with pytest.raises(da.DecodeAttnError):
        g.call(workspace=ws[:need - 256], chunk_keys=-1)


@pytest.mark.parametrize("H_Q,H_KV,B,L", [(16, 16, 3, 16384), (16, 16, 3, 16385), (32, 1, 96, 16384), (32, 1, 97, 16384)])
def test_both_sides_of_the_size_that_is_worth_sharing(H_Q, H_KV, B, L):
    """384 MiB of keys and values (768 where more than 16 heads share them) by the bound, for lengths far below it."""
    say(f"prefix bound {B} x {L}")
    Groups([(B, 300)], [40, 0, 7], H_Q, H_KV, 32, seed=23, max_pages=513).check(f"bound {B} x {L}", L=L)


@pytest.mark.parametrize("H_Q,H_KV,B,L", [(128, 1, 33, 20000), (37, 1, 64, 20000), (128, 1, 22, 4000)])
def test_a_larger_workspace_gives_the_same_bits(H_Q, H_KV, B, L):
    """Also where the one launch would write more chunk states than the call asks room for."""
    g = Groups([(B, 600)], [2000, 31], H_Q, H_KV, 32, seed=24, max_pages=625)
    need = da.da_prefix_workspace_bytes(B, 1, H_Q, H_KV)
    kv, outs = (to_dev(g.k), to_dev(g.v)), []
    for more in (0, 100, 256, 7 * need + 12):
        ws = torch.zeros(need + more, dtype=torch.uint8, device="cuda")
        say(f"prefix workspace {need} + {more}")
        lse = g.lse()
        out = g.call(lse, L=L, kv=kv, workspace=ws)
        torch.cuda.synchronize()
        outs.append((out, lse))
        assert not ws[(len(ws) & -256) - (1 << 20):].any()
    check_attention(*outs[0], g.reference(), f"bound {L}")
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(o, outs[0]))


def test_two_streams_at_once():
    g = Groups([(12, 2000)], [300, 10], 32, 4, 32, seed=22)
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = dict(kv=(to_dev(g.k), to_dev(g.v)), q=to_dev(g.q))
    want = g.call(chunk_keys=-1, **args)
    torch.cuda.synchronize()
    say("prefix on two streams")
    got = [g.call(stream=s, chunk_keys=-1, **args) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)
