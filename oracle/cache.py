"""The cache operators in float64 and plain loops: block tables from lengths,
norms and rotation, the 4-bit cache, and attention with a window and sinks.

NumPy on the CPU, from the definitions; shares no code with the HIP path."""

from __future__ import annotations

from typing import List, Optional, Tuple

import numpy as np

from .attention import bf16_bits_to_f64

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
KV4_TILE = 4352


def extend_tables(lens, new_lens, free_pages, taken, table, page, num_pages, max_tokens):
    """(table, lens_out, taken_out, cu_new, slots, positions) after the step."""
    table = table.copy()
    B, max_pages = table.shape
    lens = [max(0, int(x)) for x in lens]
    new = [max(0, int(x)) for x in new_lens]
    cu, lens_out, at = [0], [], int(taken)
    slots = np.full(max_tokens, -1, dtype=np.int32)
    positions = np.zeros(max_tokens, dtype=np.int32)
    short = False
    for b in range(B):
        row0 = cu[-1]
        cu.append(row0 + new[b])
        end = lens[b] + new[b]
        held, want = -(-lens[b] // page), -(-end // page)
        ok = end <= max_pages * page and cu[-1] <= max_tokens
        if ok and want > held:
            # requests after the first that the list could not serve get no page either
            short = short or at + want - held > len(free_pages)
            ok = not short
            if ok:
                table[b, held:want] = free_pages[at:at + want - held]
                at += want - held
        for i in range(new[b]):
            if row0 + i >= max_tokens:
                break
            pos = lens[b] + i
            positions[row0 + i] = pos
            if ok and 0 <= table[b, pos // page] < num_pages:
                slots[row0 + i] = table[b, pos // page] * page + pos % page
        lens_out.append(end if ok else lens[b])
    return table, np.array(lens_out, np.int32), at, np.array(cu, np.int32), slots, positions


def norm_rotate(x: np.ndarray, weight: Optional[np.ndarray], eps: float, rope: Optional[np.ndarray],
                positions: Optional[np.ndarray], neighbours: bool) -> Tuple[np.ndarray, np.ndarray]:
    """x float64 [N, H, D] normed and turned, and the sum of the magnitudes that make up each element."""
    y = x.astype(np.float64)
    if weight is not None:
        y = y / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + eps) * weight
    size = np.abs(y)
    if rope is None:
        return y, size
    half = rope.shape[1] // 2
    for n in range(x.shape[0]):
        inside = 0 <= positions[n] < rope.shape[0]
        for i in range(half):
            c, s = (float(rope[positions[n], i]), float(rope[positions[n], half + i])) if inside else (0.0, 0.0)
            a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
            ya, yb = y[n, :, a].copy(), y[n, :, b].copy()
            y[n, :, a], y[n, :, b] = ya * c - yb * s, yb * c + ya * s
            size[n, :, a], size[n, :, b] = abs(ya * c) + abs(yb * s), abs(yb * c) + abs(ya * s)
    return y, size


def kv4_codes(rows: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """bf16 bits [..., 128]: codes uint8 [..., 128] and scale bytes uint8 [..., 4]."""
    x = bf16_bits_to_f64(rows).reshape(rows.shape[:-1] + (4, 32))
    finite = np.isfinite(x).all(axis=-1)
    x = np.where(finite[..., None], x, 0.0)
    top = np.abs(x).max(axis=-1)
    # least e with top <= 7 * 2^e: top = f 2^x with f in [0.5, 1), 7 = 0.875 * 2^3
    f, x2 = np.frexp(top)
    e = np.clip(np.where(f <= 0.875, x2 - 3, x2 - 2), -125, 125)
    e = np.where(top == 0, -125, e)
    mag = np.abs(x) / 2.0 ** e[..., None].astype(np.float64)
    # nearest of the eight, of two equally near the even one
    code = np.zeros(mag.shape, dtype=np.int64)
    for n in range(1, 8):
        mid = (E2M1[n - 1] + E2M1[n]) / 2
        code = np.where((mag > mid) | ((mag == mid) & (n % 2 == 0)), n, code)
    code = code + 8 * np.signbit(x)
    return code.reshape(rows.shape).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def kv4_pack(k: np.ndarray, v: np.ndarray, page: int) -> np.ndarray:
    """bf16 bits [pages * page, H_KV, 128] as a 4-bit cache [pages, H_KV, page / 32, 4352]."""
    rows, H, _ = k.shape
    tiles = np.zeros((rows // 32, H, KV4_TILE), dtype=np.uint8)
    for isv, x in ((0, k), (1, v)):
        codes, scales = kv4_codes(x)
        both = codes[..., 0::2] | codes[..., 1::2] << 4
        for r in range(32):
            tiles[:, :, 2048 * isv + 64 * r:2048 * isv + 64 * r + 64] = both[r::32]
            for g in range(4):
                tiles[:, :, 4096 + 4 * (4 * (r % 16) + g) + r // 16 + 2 * isv] = scales[r::32, :, g]
    return tiles.reshape(rows // page, page // 32, H, KV4_TILE).transpose(0, 2, 1, 3).copy()


def kv4_unpack(cache: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """K and V float64 [rows, H_KV, 128] of a 4-bit cache."""
    pages, H, blocks, _ = cache.shape
    tiles = cache.transpose(0, 2, 1, 3).reshape(-1, H, KV4_TILE)
    values = np.concatenate([E2M1, -E2M1])
    out = []
    for isv in (0, 1):
        x = np.empty((tiles.shape[0], 32, H, 128))
        for r in range(32):
            both = tiles[:, :, 2048 * isv + 64 * r:2048 * isv + 64 * r + 64]
            x[:, r, :, 0::2] = values[both & 15]
            x[:, r, :, 1::2] = values[both >> 4]
            for g in range(4):
                byte = tiles[:, :, 4096 + 4 * (4 * (r % 16) + g) + r // 16 + 2 * isv].astype(np.float64)
                scale = np.where(byte == 255, np.nan, 2.0 ** (byte - 127.0))
                x[:, r, :, 32 * g:32 * g + 32] *= scale[..., None]
        out.append(x.reshape(-1, H, 128))
    return out[0], out[1]


def visible_keys(L: int, window: int, sinks: int) -> np.ndarray:
    """Positions that the query at the end of L keys sees (window 0: all)."""
    j = np.arange(L)
    return j if window == 0 else j[(j < sinks) | (j >= L - window)]


def attend(q: np.ndarray, keys: List[np.ndarray], values: List[np.ndarray],
           scale: Optional[float] = None) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """q float64 [B, H_Q, D] over each sequence's visible rows [n_b, H_KV, D]:
    (O, lse, the softmax-weighted mean of |v|, which bounds rounding errors)."""
    B, H_Q, D = q.shape
    sigma = 1.0 / np.sqrt(D) if scale is None else scale
    out, size, lse = np.zeros((B, H_Q, D)), np.zeros((B, H_Q, D)), np.full((B, H_Q), -np.inf)
    for b in range(B):
        if not len(keys[b]):
            continue
        g = H_Q // keys[b].shape[1]
        for h in range(H_Q):
            s = sigma * (keys[b][:, h // g] @ q[b, h])
            m = s.max()
            p = np.exp(s - m)
            lse[b, h] = m + np.log(p.sum())
            out[b, h] = p @ values[b][:, h // g] / p.sum()
            size[b, h] = p @ np.abs(values[b][:, h // g]) / p.sum()
    return out, lse, size
