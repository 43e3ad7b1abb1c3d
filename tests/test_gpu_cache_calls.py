"""Calls of the cache operators that their documentation allows and that are easily made: whole numbers past an
int, outputs of their own on another stream, tensors that belong to another layout."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64
from oracle.cache import kv4_unpack
from paper_2604_00028_amd import _binding as bnd
from tests.cache_helpers import Batch, check_attention, normal_bits
from tests.gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu

PAST = 2 ** 32  # wraps around to 0 in a C int


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32, device="cuda")


def refused(call, code):
    with pytest.raises(bnd.DecodeAttnError) as e:
        call()
    assert e.value.code == code


@pytest.mark.parametrize("layout", ["packed", "paged", "kv4"])
def test_numbers_past_an_int(layout):
    """Refused, not wrapped around to a batch of 100 keys, to one split or to no packing."""
    batch = Batch([300, 20], 8, 2, layout, seed=1)
    call = batch.call_kv4 if layout == "kv4" else batch.call_window
    say(f"numbers past an int {layout}")
    refused(lambda: call(da, 50, 0, L=PAST + 100), bnd.DA_ERR_SHAPE)
    refused(lambda: call(da, 50, 0, num_splits=PAST + 1), bnd.DA_ERR_SPLITS)
    refused(lambda: call(da, -PAST + 50, 0), bnd.DA_ERR_ARG)
    refused(lambda: call(da, 50, -PAST), bnd.DA_ERR_ARG)
    if layout != "kv4":
        refused(lambda: call(da, 50, 0, pack_gqa=PAST), bnd.DA_ERR_ARG)


def test_numbers_past_an_int_without_a_window():
    batch = Batch([300, 20], 8, 2, "packed", seed=1)
    q, k, v, cu = to_dev(batch.q), to_dev(batch.k), to_dev(batch.v), torch.from_numpy(batch.cu).cuda()
    paged = Batch([300, 20], 8, 2, "paged", seed=1)
    pk, pv, table = to_dev(paged.k), to_dev(paged.v), torch.from_numpy(paged.table).cuda()
    say("numbers past an int, no window")
    for call in (da.da_decode_attn, da.da_decode_attn_noalloc):
        refused(lambda: call(q, k, v, cu, L_K_max=PAST + 100), bnd.DA_ERR_SHAPE)
        refused(lambda: call(q, k, v, cu, L_K_max=300, num_splits=PAST + 1), bnd.DA_ERR_SPLITS)
    refused(lambda: da.da_decode_attn_dealt(q, k, v, PAST + 100, cu), bnd.DA_ERR_SHAPE)
    refused(lambda: da.da_decode_attn_paged(q, pk, pv, table, paged.seq_lens(), PAST + 100), bnd.DA_ERR_SHAPE)


def test_tables_past_an_int():
    say("tables past an int")

    def tables(page, pages, rows=8):
        return da.da_extend_tables(ints(2), ints(2), ints(4), ints(1), ints(2, 4), page, pages, rows)

    tables(16, 9)
    refused(lambda: tables(PAST + 16, 9), bnd.DA_ERR_SHAPE)
    refused(lambda: tables(-PAST + 16, 9), bnd.DA_ERR_SHAPE)
    refused(lambda: tables(16, PAST + 9), bnd.DA_ERR_SHAPE)
    for rows in (PAST + 8, 2 ** 28 + 1, -1):
        with pytest.raises(ValueError):
            tables(16, 9, rows)


def calls_with_outputs():
    """name -> call(stream): entry points that make their own outputs, over inputs that stay."""
    rng = np.random.default_rng(3)
    packed, paged, four = (Batch([3000, 200, 1], 8, 2, layout, seed=3) for layout in ("packed", "paged", "kv4"))
    q, k, v, cu = to_dev(packed.q), to_dev(packed.k), to_dev(packed.v), torch.from_numpy(packed.cu).cuda()
    pk, pv, table, lens = to_dev(paged.k), to_dev(paged.v), torch.from_numpy(paged.table).cuda(), paged.seq_lens()
    cache, table4 = torch.from_numpy(four.cache).cuda(), torch.from_numpy(four.table).cuda()
    x = to_dev(normal_bits(rng, (40, 12, 128)))
    parts = x[:, :8], x[:, 8:10], x[:, 10:]
    rows = torch.zeros(2, 64, 2, 128, dtype=torch.bfloat16, device="cuda")
    spare = torch.zeros(2, 2, 1, 4352, dtype=torch.uint8, device="cuda")
    tables = [torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([5, 9], [30, 2], [3, 1, 0, 2], [0])]
    entries, cu_new = ints(2, 4), ints(3)
    L = 3000
    states = lambda s: da.da_split_partials(q, k, v, cu, num_splits=4, pack_gqa=1, L_K_max=L, stream=s)  # noqa: E731
    held = states(None)
    plan = da.da_make_plan(3, 8, 2, L, num_splits=4)
    sched, meta = da.da_make_schedule(packed.lengths, 8, 2)
    meta = meta.cuda()
    return {
        "tables": lambda s: da.da_extend_tables(*tables, entries, 16, 9, 40, stream=s),
        "tables, some given": lambda s: da.da_extend_tables(*tables, entries, 16, 9, 40, cu_new=cu_new, stream=s),
        "append": lambda s: da.da_append_kv(*parts, None, None, *rows, stream=s),
        "append4": lambda s: da.da_append_kv4(*parts, None, None, spare, stream=s),
        "read4": lambda s: da.da_read_kv4(cache, stream=s),
        "window": lambda s: da.da_decode_attn_window(q, pk, pv, 500, 4, None, table, lens, L_K_max=L, stream=s),
        "kv4": lambda s: da.da_decode_attn_kv4(q, cache, table4, lens, L, stream=s),
        "plain": lambda s: da.da_decode_attn(q, k, v, cu, L_K_max=L, num_splits=4, stream=s),
        "planned": lambda s: da.da_decode_attn_planned(q, k, v, plan, cu, L_K_max=L, stream=s),
        "noalloc": lambda s: da.da_decode_attn_noalloc(q, k, v, cu, L_K_max=L, stream=s),
        "paged": lambda s: da.da_decode_attn_paged(q, pk, pv, table, lens, L, num_splits=4, stream=s),
        "paged planned": lambda s: da.da_decode_attn_paged_planned(q, pk, pv, table, lens, L, plan, stream=s),
        "dealt": lambda s: da.da_decode_attn_dealt(q, k, v, L, cu, stream=s),
        "scheduled": lambda s: da.da_decode_attn_scheduled(q, k, v, sched, meta, cu, stream=s),
        "partials": states,
        "merge": lambda s: da.da_combine_splits(*held, stream=s),
    }


def test_outputs_of_calls_on_another_stream():
    """Memory that the current stream has freed, but whose last work it still has to do, is none for the
    outputs of a call on another stream."""
    side = torch.cuda.Stream()
    a = torch.randn(8192, 8192, device="cuda").bfloat16()
    product = torch.empty_like(a)
    for name, call in calls_with_outputs().items():
        say(f"own outputs on another stream: {name}")
        listed = lambda out: list(out) if isinstance(out, (tuple, list)) else [out]  # noqa: E731
        torch.mm(a, a, out=product)
        call(side)  # its workspace, which waits for the current stream where it is new
        torch.cuda.synchronize()
        want = [t.clone() for t in listed(call(None))]
        freed = [torch.empty_like(t) for t in want]
        torch.cuda.synchronize()
        for _ in range(20):  # some 15 ms
            torch.mm(a, a, out=product)
        for t in freed:
            t.fill_(7)
        del freed, t
        got = listed(call(side))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w), name


def test_a_workspace_the_gpu_cannot_write_is_refused():
    batch, four = Batch([3000, 200], 8, 2, "packed", seed=4), Batch([3000, 200], 8, 2, "kv4", seed=4)
    q, k, v, cu = to_dev(batch.q), to_dev(batch.k), to_dev(batch.v), torch.from_numpy(batch.cu).cuda()
    plan = da.da_make_plan(2, 8, 2, 3000, num_splits=4)
    for ws in (torch.zeros(8 << 20, dtype=torch.uint8), torch.zeros(16 << 20, dtype=torch.uint8, device="cuda")[::2]):
        say(f"workspace on {ws.device}, contiguous {ws.is_contiguous()}")
        for call in (lambda: batch.call_window(da, 2000, 4, num_splits=4, workspace=ws),
                     lambda: four.call_kv4(da, num_splits=4, workspace=ws),
                     lambda: da.da_decode_attn(q, k, v, cu, L_K_max=3000, num_splits=4, workspace=ws),
                     lambda: da.da_decode_attn_planned(q, k, v, plan, cu, L_K_max=3000, workspace=ws),
                     lambda: da.da_decode_attn_dealt(q, k, v, 3000, cu, workspace=ws)):
            with pytest.raises(ValueError):
                call()


def test_lengths_of_another_layout_are_refused():
    """A padded dense batch with seq_lens would be attended to its full length, a paged one with
    cu_seqlens_k by its seq_lens."""
    dense, paged = Batch([64, 64], 8, 2, "dense", seed=5), Batch([64, 30], 8, 2, "paged", seed=5)
    cu = torch.tensor([0, 64, 94], dtype=torch.int32, device="cuda")
    say("lengths of another layout")
    dense.call_window(da, 50, 4)
    paged.call_window(da, 50, 4)
    with pytest.raises(ValueError):
        dense.call_window(da, 50, 4, seq_lens=paged.seq_lens())
    with pytest.raises(ValueError):
        paged.call_window(da, 50, 4, cu_seqlens_k=cu)


@pytest.mark.parametrize("H_Q,H_KV,L", [(16, 8, (1 << 20) + 77), (16, 16, (1 << 19) + 1), (8, 1, (1 << 23) + 40)])
def test_four_bit_sequences_of_two_gib_of_bf16_keys_and_more(H_Q, H_KV, L):
    """The 4-bit cache is addressed by page, so no product of length and heads bounds it.  The sequence is one page
    of distinct keys again and again: each counts as often as it comes, in the sums and in the log-sum-exp.

    At most 1024 steps of 64 keys a wave, whose sums take one rounding of 2^-24 a step (2^-14 of l) and the outputs
    two (2^-13 of the weighted mean of |v|): within what check_attention allows (2^-13 of lse, 2^-12)."""
    page = 512
    batch = Batch([page], H_Q, H_KV, "kv4", page=page, seed=H_KV, max_pages=1)
    k, v = (x[batch.rows[0]] for x in kv4_unpack(batch.cache))
    pages = -(-L // page)
    table = torch.full((1, pages), int(batch.table[0, 0]), dtype=torch.int32, device="cuda")
    lens = torch.tensor([L], dtype=torch.int32, device="cuda")
    q, cache = to_dev(batch.q), torch.from_numpy(batch.cache).cuda()
    times = np.where(np.arange(page) < L % page, L // page + 1, L // page).astype(np.float64)
    s = np.einsum("hd,khd->hk", bf16_bits_to_f64(batch.q)[0], k.repeat(H_Q // H_KV, 1)) / np.sqrt(128.0)
    top = s.max(1, keepdims=True)
    p = np.exp(s - top) * times
    lse = (top[:, 0] + np.log(p.sum(1)))[None]
    p /= p.sum(1, keepdims=True)
    v = v.repeat(H_Q // H_KV, 1)
    ref = np.einsum("hk,khd->hd", p, v)[None], lse, np.einsum("hk,khd->hd", p, np.abs(v))[None]
    for splits in (0, 64):
        got = torch.empty(1, H_Q, dtype=torch.float32, device="cuda")
        say(f"long 4-bit sequence {H_Q}/{H_KV} L={L} splits={splits}")
        out = da.da_decode_attn_kv4(q, cache, table, lens, L, lse_out=got, num_splits=splits)
        torch.cuda.synchronize()
        check_attention(out, got, ref, f"{H_Q}/{H_KV} L={L}")
