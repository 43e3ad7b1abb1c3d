"""Calls of the cache operators that their documentation allows and that are easily made: whole numbers past an
int, outputs of their own on another stream, tensors that belong to another layout."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from paper_2604_00028_amd import _binding as bnd
from tests.cache_helpers import Batch
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
    tables = lambda page, pages, rows=8: da.da_extend_tables(ints(2), ints(2), ints(4), ints(1), ints(2, 4),  # noqa: E731
                                                             page, pages, rows)
    tables(16, 9)
    refused(lambda: tables(PAST + 16, 9), bnd.DA_ERR_SHAPE)
    refused(lambda: tables(-PAST + 16, 9), bnd.DA_ERR_SHAPE)
    refused(lambda: tables(16, PAST + 9), bnd.DA_ERR_SHAPE)
    for rows in (PAST + 8, 2 ** 28 + 1, -1):
        with pytest.raises(ValueError):
            tables(16, 9, rows)
