"""Keys whose scores are -inf weigh nothing in any attention call, also where a wave or a chunk begins with them."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from tests.cache_helpers import Batch, check_attention, new_lse
from tests.gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu


def batch(layout, H_Q, H_KV):
    """The first ten tiles of each sequence at -inf for every head, and all but the last key of one."""
    lengths = [700, 700, 700] if layout == "dense" else [700, 1100, 430]
    b = Batch(lengths, H_Q, H_KV, layout, 32, seed=51)
    b.q[:, :, 7] = 0x3F80  # 1
    for i, rows in enumerate(b.rows):
        dead = rows[:320] if i != 2 else rows[:-1]
        b.k.reshape(-1, H_KV, 128)[dead, :, 7] = 0xFF80
    return b


def calls(b):
    """The attention calls of the layout, by name."""
    q, k, v = to_dev(b.q), to_dev(b.k), to_dev(b.v)
    out = {"window": lambda lse: b.call_window(da, 10 ** 6, 0, lse)}
    if b.layout == "paged":
        table, lens = torch.from_numpy(b.table).cuda(), b.seq_lens()
        for s in (0, 1, 2, 9):
            out[f"paged, {s} splits"] = lambda lse, s=s: da.da_decode_attn_paged(q, k, v, table, lens, b.L, lse_out=lse,
                                                                                num_splits=s)
        out["dealt"] = lambda lse: da.da_decode_attn_dealt(q, k, v, b.L, block_table=table, seq_lens=lens, lse_out=lse)
        return out
    cu = torch.from_numpy(b.cu).cuda() if b.layout == "packed" else None
    for s in (0, 1, 2, 9):
        for pack in (-1, 0):
            out[f"{s} splits, pack {pack}"] = lambda lse, s=s, pack=pack: da.da_decode_attn(
                q, k, v, cu, lse_out=lse, L_K_max=b.L, num_splits=s, pack_gqa=pack)
    if b.layout == "packed":
        out["dealt"] = lambda lse: da.da_decode_attn_dealt(q, k, v, b.L, cu, lse_out=lse)
        sched, meta = da.da_make_schedule(b.lengths, b.q.shape[1], b.H_KV, b.L)
        out["scheduled"] = lambda lse: da.da_decode_attn_scheduled(q, k, v, sched, meta.cuda(), cu, lse_out=lse)
    return out


@pytest.mark.parametrize("H_Q,H_KV", [(16, 2), (32, 1), (4, 4)])
@pytest.mark.parametrize("layout", ["dense", "packed", "paged"])
def test_every_call(layout, H_Q, H_KV):
    b = batch(layout, H_Q, H_KV)
    ref = b.reference(0, 0)
    for name, call in calls(b).items():
        say(f"scores of -inf, {layout} {H_Q}/{H_KV}: {name}")
        lse = new_lse(b)
        out = call(lse)
        torch.cuda.synchronize()
        check_attention(out, lse, ref, f"{layout} {name}")


def test_a_chunk_of_nothing_else_is_an_empty_one():
    b = batch("dense", 16, 2)
    say("scores of -inf, chunk states")
    o, m, l = da.da_split_partials(to_dev(b.q), to_dev(b.k), to_dev(b.v), num_splits=7, pack_gqa=1)
    torch.cuda.synchronize()
    assert (l[:3] == 0).all() and torch.isneginf(m[:3]).all() and (o[:3] == 0).all()  # the first 300 keys
    assert np.isfinite(o.cpu().numpy()).all() and (l[6] > 0).all()
