"""The cache operators on the CPU: refusals (every call below returns before any
HIP call), host-side sizing, and the oracle they are tested against."""

import numpy as np
import pytest
import torch

import paper_2604_00028_amd as da
from oracle import bf16_bits_to_f64, decode_attention
from oracle.cache import (attend, extend_tables, kv4_codes, kv4_pack, kv4_unpack, norm_rotate, visible_keys)
from paper_2604_00028_amd import _binding as bnd
from workloads import f32_to_bf16_bits

FAKE = 0x100000  # 16-byte aligned stand-in device address (never dereferenced)
NULL, SHAPE, UNSUP, SPLITS, ALIGN, WS, ARG = (bnd.DA_ERR_NULL, bnd.DA_ERR_SHAPE, bnd.DA_ERR_UNSUPPORTED,
                                              bnd.DA_ERR_SPLITS, bnd.DA_ERR_ALIGN, bnd.DA_ERR_WORKSPACE,
                                              bnd.DA_ERR_ARG)


def refused(rc, code):
    assert rc == code
    assert da.da_last_error() != ""


def window(lib, q=FAKE, k=FAKE, v=FAKE, cu=None, table=FAKE, lens=FAKE, page=64, max_pages=32, pages=64, out=FAKE,
           lse=None, B=2, H_Q=8, H_KV=1, L=2048, d=128, window=100, sinks=4, s=1, pack=-1, ws=None, ws_bytes=0):
    return lib.da_decode_attn_window(q, k, v, cu, table, lens, page, max_pages, pages, out, lse, B, H_Q, H_KV, L, d, 0.0,
                                     window, sinks, s, pack, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(out=None), NULL), (dict(lens=None), NULL),
    (dict(table=None, k=None), NULL), (dict(B=0), SHAPE), (dict(H_Q=9, H_KV=2), SHAPE), (dict(L=-1), SHAPE),
    (dict(max_pages=31), SHAPE), (dict(table=None, L=1 << 23), SHAPE), (dict(d=64), UNSUP), (dict(page=48), UNSUP),
    (dict(page=0), UNSUP), (dict(window=0), ARG), (dict(window=-5), ARG), (dict(sinks=-1), ARG), (dict(pack=3), ARG),
    (dict(s=65), SPLITS), (dict(q=FAKE + 8), ALIGN), (dict(k=FAKE + 2), ALIGN), (dict(out=FAKE + 4), ALIGN),
    (dict(table=FAKE + 2), ALIGN), (dict(lens=FAKE + 1), ALIGN), (dict(lse=FAKE + 2), ALIGN),
    (dict(table=None, cu=FAKE + 2), ALIGN), (dict(s=4), WS), (dict(s=4, ws=FAKE, ws_bytes=1000), WS),
    (dict(s=4, ws=FAKE + 4, ws_bytes=1 << 30), ALIGN),
])
def test_window_refusals(lib, kw, code):
    refused(window(lib, **kw), code)


def kv4(lib, q=FAKE, cache=FAKE, table=FAKE, lens=FAKE, out=FAKE, lse=None, B=2, H_Q=8, H_KV=1, page=64, max_pages=32,
        pages=64, L=2048, d=128, window=0, sinks=0, s=0, ws=None, ws_bytes=0):
    return lib.da_decode_attn_kv4(q, cache, table, lens, out, lse, B, H_Q, H_KV, page, max_pages, pages, L, d, 0.0, window,
                                  sinks, s, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(cache=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL),
    (dict(out=None), NULL), (dict(B=-1), SHAPE), (dict(H_Q=9, H_KV=2), SHAPE), (dict(max_pages=31), SHAPE),
    (dict(pages=-1), SHAPE), (dict(H_KV=64, H_Q=64, page=1 << 20, max_pages=1), SHAPE), (dict(d=256), UNSUP),
    (dict(page=16), UNSUP), (dict(page=1 << 21), UNSUP), (dict(window=-1), ARG), (dict(sinks=-1), ARG),
    (dict(s=65), SPLITS), (dict(q=FAKE + 2), ALIGN), (dict(cache=FAKE + 4), ALIGN), (dict(out=FAKE + 8), ALIGN),
    (dict(lens=FAKE + 2), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(lse=FAKE + 1), ALIGN),
    (dict(ws=FAKE + 8, ws_bytes=1 << 30), ALIGN),
])
def test_kv4_refusals(lib, kw, code):
    refused(kv4(lib, **kw), code)


def append(lib, four, q=FAKE, qs=1024, k=FAKE, ks=128, v=FAKE, vs=128, wq=FAKE, wk=FAKE, eps=1e-6, rope=FAKE, rows=10,
           rot=128, nb=0, pos=FAKE, slots=FAKE, out=FAKE, kc=FAKE, vc=FAKE, num_rows=100, page=32, pages=4, N=3, H_Q=8,
           H_KV=1, d=128):
    head = (q, qs, k, ks, v, vs, wq, wk, eps, rope, rows, rot, nb, pos, slots, out)
    if four:
        return lib.da_append_kv4(*head, kc, page, pages, N, H_Q, H_KV, d, None)
    return lib.da_append_kv(*head, kc, vc, num_rows, N, H_Q, H_KV, d, None)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(q=None), NULL), (dict(H_Q=0), NULL), (dict(out=None), NULL),
    (dict(pos=None), NULL), (dict(kc=None), NULL), (dict(N=-1), SHAPE), (dict(H_KV=0), SHAPE), (dict(H_Q=-1), SHAPE),
    (dict(N=1 << 25), SHAPE), (dict(rows=0), SHAPE), (dict(d=64), UNSUP), (dict(rot=144), UNSUP), (dict(rot=8), UNSUP),
    (dict(rot=40), UNSUP), (dict(nb=2), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG),
    (dict(q=FAKE + 2), ALIGN), (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 4), ALIGN), (dict(out=FAKE + 8), ALIGN),
    (dict(wq=FAKE + 2), ALIGN), (dict(wk=FAKE + 8), ALIGN), (dict(rope=FAKE + 4), ALIGN), (dict(pos=FAKE + 2), ALIGN),
    (dict(slots=FAKE + 1), ALIGN), (dict(kc=FAKE + 2), ALIGN), (dict(qs=1028), ALIGN), (dict(ks=-128), ALIGN),
    (dict(vs=4), ALIGN),
])
def test_append_refusals(lib, four, kw, code):
    refused(append(lib, four, **kw), code)


@pytest.mark.parametrize("four,kw,code", [
    (False, dict(vc=None), NULL), (False, dict(num_rows=-1), SHAPE), (False, dict(vc=FAKE + 2), ALIGN),
    (True, dict(page=33), UNSUP), (True, dict(pages=-1), SHAPE), (True, dict(page=1 << 20, pages=1 << 11), SHAPE),
])
def test_append_cache_refusals(lib, four, kw, code):
    refused(append(lib, four, **kw), code)


def read(lib, cache=FAKE, slots=None, k=FAKE, v=FAKE, N=3, H_KV=1, page=32, pages=4, d=128):
    return lib.da_read_kv4(cache, slots, k, v, N, H_KV, page, pages, d, None)


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(N=-1), SHAPE), (dict(N=1 << 27), SHAPE),
    (dict(H_KV=0), SHAPE), (dict(pages=-2), SHAPE), (dict(page=20), UNSUP), (dict(d=127), UNSUP),
    (dict(cache=FAKE + 8), ALIGN), (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 2), ALIGN), (dict(slots=FAKE + 2), ALIGN),
])
def test_read_refusals(lib, kw, code):
    refused(read(lib, **kw), code)


def tables(lib, lens=FAKE, new=FAKE, free=FAKE, taken=FAKE, table=FAKE, lens_out=FAKE, taken_out=FAKE, cu=FAKE,
           slots=FAKE, pos=FAKE, B=2, page=16, max_pages=8, pages=100, num_free=10, tokens=20):
    return lib.da_extend_tables(lens, new, free, taken, table, lens_out, taken_out, cu, slots, pos, B, page, max_pages,
                                pages, num_free, tokens, None)


@pytest.mark.parametrize("kw,code", [
    (dict(lens=None), NULL), (dict(new=None), NULL), (dict(free=None), NULL), (dict(taken=None), NULL),
    (dict(table=None), NULL), (dict(lens_out=None), NULL), (dict(taken_out=None), NULL), (dict(slots=None), NULL),
    (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(page=0), SHAPE), (dict(page=(1 << 20) + 1), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(pages=-1), SHAPE), (dict(num_free=-1), SHAPE), (dict(num_free=1 << 30), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(tokens=(1 << 28) + 1), SHAPE), (dict(page=1 << 20, pages=1 << 11), SHAPE),
    (dict(lens=FAKE + 2), ALIGN), (dict(slots=FAKE + 1), ALIGN), (dict(pos=FAKE + 2), ALIGN), (dict(cu=FAKE + 3), ALIGN),
])
def test_table_refusals(lib, kw, code):
    refused(tables(lib, **kw), code)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would run")
def test_calls_that_pass_the_checks_reach_the_device_check(lib):
    """No GPU here: a call with nothing to refuse ends at the device query."""
    for rc in (window(lib), kv4(lib), append(lib, False), append(lib, True), append(lib, False, q=None, H_Q=0, rope=None,
               pos=None, wq=None, wk=None, slots=None), read(lib), tables(lib), tables(lib, cu=None, pos=None)):
        assert rc in (bnd.DA_ERR_HIP, UNSUP)


def test_binding_refuses_tensors_that_do_not_fit():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)    # noqa: E731
    with pytest.raises(ValueError):
        da.da_decode_attn_window(bf(1, 8, 128), bf(1, 64, 1, 128), bf(1, 64, 1, 128), 16)
    with pytest.raises(ValueError):
        da.da_decode_attn_kv4(bf(1, 8, 128), torch.zeros(2, 1, 1, 4352, dtype=torch.uint8), i32(1, 1), i32(1), 32)
    with pytest.raises(ValueError):
        da.da_append_kv(bf(1, 8, 128), bf(1, 1, 128), bf(1, 1, 128), None, None, bf(4, 1, 128), bf(4, 1, 128))
    with pytest.raises(ValueError):
        da.da_read_kv4(torch.zeros(2, 1, 1, 4352, dtype=torch.uint8))
    with pytest.raises(ValueError):
        da.da_extend_tables(i32(2), i32(2), i32(4), i32(1), i32(2, 4), 16, 8, 2)


def test_window_keys(lib):
    assert da.da_window_keys(10000, 1, 0) == 32
    assert da.da_window_keys(10000, 32, 0) == 64       # a window of 32 may touch two tiles
    assert da.da_window_keys(10000, 34, 0) == 96       # and one of 34 three
    assert da.da_window_keys(10000, 33, 33) == 64 + 64
    assert da.da_window_keys(50, 100, 4) == 50
    assert da.da_window_keys(100, 2 ** 31 - 1, 2 ** 31 - 1) == 100
    assert da.da_window_keys(0, 5, 0) == 0
    for bad in ((-1, 5, 0), (10, 0, 0), (10, 5, -1)):
        assert da.da_window_keys(*bad) == -1
    rng = np.random.default_rng(0)
    for _ in range(300):                               # tiles that hold a visible key, counted
        L, W, S = (int(rng.integers(1, n)) for n in (2000, 500, 200))
        tiles = len({int(j) // 32 for j in visible_keys(L, W, S)})
        assert 32 * (tiles - 1) < da.da_window_keys(L, W, S) and tiles * 32 <= da.da_window_keys(L, W, S) + 31


def test_kv4_workspace(lib):
    size = lambda *a, **k: da.da_kv4_workspace_bytes(*a, num_cus=256, **k)  # noqa: E731
    assert size(1, 64, 8, 128) == 0 and size(1, 64, 8, 8192, num_splits=1) == 0
    need = size(1, 64, 8, 8192, num_splits=4)
    assert need == da.da_workspace_bytes(1, 64, 128, 4)
    # an unknown pool is enough for any
    for B in (1, 3, 40):
        for keys in (64, 5000, 10 ** 6, 10 ** 9):
            assert size(B, 64, 8, 30000, 0) >= size(B, 64, 8, 30000, keys)
    assert size(0, 64, 8, 128) == 0 and size(1, 64, 8, 128, window=-1) == 0 and size(1, 64, 8, 128, num_splits=65) == 0
    assert size(1, 64, 8, 1 << 20, 0, 64, 4) == 0      # a window of a few tiles is one chunk


# ---------------------------------------------------------------- the oracle


def test_oracle_codes_against_the_bits():
    """Codes and scales decoded by their bit fields give the nearest value there is, and the scale is the least."""
    rng = np.random.default_rng(1)
    x = f32_to_bf16_bits(rng.standard_normal((40, 128)).astype(np.float32) * 10.0 ** rng.integers(-5, 5, (40, 1)))
    codes, scales = kv4_codes(x)
    f = bf16_bits_to_f64(x).reshape(40, 4, 32)
    e, m = (codes >> 1) & 3, codes & 1
    mag = np.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e.astype(float) - 1))
    got = (np.where(codes >= 8, -mag, mag).reshape(40, 4, 32)) * 2.0 ** (scales[..., None].astype(float) - 127)
    top = np.abs(f).max(-1)
    unit = 2.0 ** (scales.astype(float) - 127)
    assert np.all(top <= 7 * unit) and np.all(top > 3.5 * unit)
    grid = np.array([s * v for v in (0, 0.5, 1, 1.5, 2, 3, 4, 6) for s in (1, -1)])
    best = np.abs(f[..., None] - grid * unit[..., None, None]).min(-1)
    assert np.array_equal(np.abs(f - got), best)


def test_oracle_pack_round_trip_and_ties():
    rng = np.random.default_rng(2)
    k, v = (f32_to_bf16_bits(rng.standard_normal((96, 3, 128)).astype(np.float32)) for _ in range(2))
    ku, vu = kv4_unpack(kv4_pack(k, v, 96))
    again = kv4_unpack(kv4_pack(f32_to_bf16_bits(ku.astype(np.float32)), f32_to_bf16_bits(vu.astype(np.float32)), 32))
    assert np.array_equal(again[0], ku) and np.array_equal(again[1], vu)      # values there are stay
    row = np.zeros((1, 128), np.float32)
    row[0, :9] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5]
    codes, scales = kv4_codes(f32_to_bf16_bits(row))
    assert codes[0, :9].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 14] and scales[0, 0] == 127


def test_oracle_window_and_attention():
    assert visible_keys(10, 3, 2).tolist() == [0, 1, 7, 8, 9]
    assert visible_keys(4, 3, 2).tolist() == [0, 1, 2, 3]
    assert visible_keys(0, 3, 2).tolist() == [] and visible_keys(5, 0, 2).tolist() == [0, 1, 2, 3, 4]
    rng = np.random.default_rng(3)
    q, k, v = (f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32))
               for s in ((2, 4, 128), (2, 50, 2, 128), (2, 50, 2, 128)))
    want, want_lse = decode_attention(q, k, v)
    got, lse, size = attend(bf16_bits_to_f64(q), list(bf16_bits_to_f64(k)), list(bf16_bits_to_f64(v)))
    assert np.allclose(got, want, rtol=1e-12, atol=1e-14) and np.allclose(lse, want_lse, rtol=1e-13)
    assert np.all(size >= np.abs(got) - 1e-14)


@pytest.mark.parametrize("neighbours", [False, True])
def test_oracle_rotation_is_one(neighbours):
    """Lengths of pairs stay, equal positions turn by equal angles (inner products depend on their difference)."""
    rng = np.random.default_rng(4)
    x, y = rng.standard_normal((2, 1, 1, 128))
    ang = np.arange(40)[:, None] * 0.1 ** (np.arange(32) / 32)
    rope = np.concatenate([np.cos(ang), np.sin(ang)], 1)
    turn = lambda z, p: norm_rotate(z, None, 0.0, rope, [p], neighbours)[0]  # noqa: E731
    assert np.isclose(np.linalg.norm(turn(x, 17)), np.linalg.norm(x)) and np.array_equal(turn(x, 0), x)
    assert np.isclose((turn(x, 20) * turn(y, 13)).sum(), (turn(x, 9) * turn(y, 2)).sum())
    w = rng.standard_normal(128)
    normed = norm_rotate(x, w, 0.0, None, None, neighbours)[0]
    assert np.isclose(np.sqrt(np.mean((normed / w) ** 2)), 1.0)
    assert np.all(norm_rotate(x, None, 0.0, rope, [40], neighbours)[0][..., :64] == 0)  # outside the table


def test_oracle_tables_give_every_page_once():
    rng = np.random.default_rng(5)
    page, B = 8, 30
    lens, taken = np.zeros(B, int), 0
    free = rng.permutation(200)
    table = np.full((B, 20), -1, np.int32)
    owned = set()
    for step in range(30):
        new = rng.integers(0, 9, B)
        before = lens
        table, lens, taken, cu, slots, pos = extend_tables(lens, new, free, taken, table, page, 200, 400)
        assert np.all((lens == before + new) | (lens == before)) and cu[-1] == new.sum()
        live = slots[slots >= 0].tolist()
        assert len(set(live)) == len(live) == int((lens - before).sum()) and not owned & set(live)
        owned |= set(live)
        used = [int(p) for b in range(B) for p in table[b, :-(-lens[b] // page)]]
        assert len(used) == len(set(used)) == taken and set(used) == set(free[:taken].tolist())
    assert taken > 190  # the list ran out on the way


def test_windows_past_an_int_are_windows_over_everything():
    assert da.da_window_keys(1000, 2 ** 40) == da.da_window_keys(1000, 2 ** 31 - 1) == 1000
    assert da.da_window_keys(1000, 5, 2 ** 40) == 1000
    sizes = [da.da_kv4_workspace_bytes(4, 64, 8, 4000, 0, w, s, 8, 256) for w, s in ((0, 0), (2 ** 40, 0), (5, 2 ** 33))]
    assert sizes[0] > 0 and sizes[0] == sizes[1] == sizes[2]
