"""The calls around a decode step's cache, as cases that can be timed and
checked: what a server does between the projections and the attention's
output.

Each case is one `op` with its sizes:

  tables   da_extend_tables: request lengths grow; block tables, slots and positions follow
  append   da_append_kv: norms of q and k per head, rotation, rows into a bf16 cache
  append4  da_append_kv4 and da_read_kv4: rows into a cache of 4-bit values, and the cache read back
  window   da_decode_attn_window: one query token per sequence, the last `window` keys and the first `sinks` visible
  kv4      da_decode_attn_kv4: one query token per sequence over a paged cache of 4-bit values

With `own` false, run() computes the same in elementary torch operations in 32
bits.  Lengths of a batch follow from the case alone (`lens`, `len_lo`,
`len_hi`, `len_seed`), so its work is known; the seed of prepare() draws the
tensors, the order of pages and of requests.

The 4-bit cache is uint8 [num_pages, H_KV, page / 32, 4352]: for 32 keys of
one head, 32 x 64 bytes of K codes, as many of V, then 256 scale bytes.  Byte
i of a row holds dims 2i (low) and 2i + 1; the scale of block g (32 dims) of
key r sits at 4 * (4 * (r % 16) + g) + r / 16, two further on for V.
"""

import math

import numpy as np
import torch

own = False

D = 128
DEV = "cuda"
EPS = 1e-6
TILE = 32            # keys per block of the 4-bit cache
TILE_BYTES = 4352
# (query heads, KV heads): MQA, GQA groups of 4 to 64, and no sharing
HEADS = [(8, 1), (32, 1), (16, 2), (32, 2), (128, 2), (32, 4), (64, 4), (64, 8), (40, 8), (128, 16), (16, 16)]
MAX_KV_BYTES = 1 << 30     # bf16 bytes of the keys a drawn attention case sees
MAX_PADDED = 4 << 30       # the same with every sequence padded to the longest
MAX_TOKEN_HEADS = 8192 * 80


def listed():
    return [
        # a decode step of 64 requests, one new token each: bound by launch and latency
        {"name": "tables_decode_b64", "op": "tables", "B": 64, "new": "one", "page": 64,
         "lens": "lognormal", "len_lo": 16, "len_hi": 32768, "len_seed": 31, "pool": 1.25},
        # a loaded server's step: 500 requests, most decode, some bring prompt pieces; the free list runs short
        {"name": "tables_mixed_b500", "op": "tables", "B": 500, "new": "mixed", "page": 32,
         "lens": "lognormal", "len_lo": 0, "len_hi": 16384, "len_seed": 32, "pool": 0.95},
        # one decode token of Llama-3.1-70B's heads
        {"name": "append_n1", "op": "append", "N": 1, "H_Q": 64, "H_KV": 8, "page": 64, "rot": 128, "pairs": "halves",
         "norm": True, "far": 8192},
        # a decode batch of 61 tokens at far positions, half of each head rotated in neighbouring pairs
        {"name": "append_n61_pairs", "op": "append", "N": 61, "H_Q": 32, "H_KV": 4, "page": 32, "rot": 64,
         "pairs": "neighbours", "norm": True, "far": 131072},
        # a prompt of 8192 tokens
        {"name": "append_n8192", "op": "append", "N": 8192, "H_Q": 64, "H_KV": 8, "page": 64, "rot": 128,
         "pairs": "halves", "norm": True, "far": 8192},
        # a prompt piece of odd length into the 4-bit cache, and the cache read back for a shared prefix
        {"name": "append4_n3001", "op": "append4", "N": 3001, "H_KV": 8, "page": 64},
        # one long context, a window of 512 and 4 sinks: bound by latency
        {"name": "window_b1_w512", "op": "window", "layout": "paged", "B": 1, "H_Q": 64, "H_KV": 8, "page": 64,
         "lens": "uniform", "len_lo": 8191, "len_hi": 8191, "len_seed": 1, "window": 512, "sinks": 4},
        # pure MQA, a packed batch of odd lengths around the window
        {"name": "window_mqa_b16_w1000", "op": "window", "layout": "packed", "B": 16, "H_Q": 32, "H_KV": 1,
         "lens": "uniform", "len_lo": 33, "len_hi": 8000, "len_seed": 41, "window": 1000, "sinks": 0},
        # a loaded server: 32 long contexts, a window of 4096 and 64 sinks
        {"name": "window_b32_w4096", "op": "window", "layout": "paged", "B": 32, "H_Q": 64, "H_KV": 8, "page": 64,
         "lens": "uniform", "len_lo": 6000, "len_hi": 12000, "len_seed": 42, "window": 4096, "sinks": 64},
        # one context of 4001 keys in 4 bits
        {"name": "kv4_b1_l4001", "op": "kv4", "B": 1, "H_Q": 64, "H_KV": 8, "page": 64,
         "lens": "uniform", "len_lo": 4001, "len_hi": 4001, "len_seed": 1, "window": 0, "sinks": 0},
        # most sequences short, a few long, in 4 bits
        {"name": "kv4_b64_lognormal", "op": "kv4", "B": 64, "H_Q": 32, "H_KV": 4, "page": 64,
         "lens": "lognormal", "len_lo": 16, "len_hi": 32768, "len_seed": 102, "window": 0, "sinks": 0},
        # the largest: 32 sequences of 8192 keys in 4 bits, 285 MB of cache
        {"name": "kv4_b32_l8192", "op": "kv4", "B": 32, "H_Q": 64, "H_KV": 8, "page": 128,
         "lens": "uniform", "len_lo": 8192, "len_hi": 8192, "len_seed": 1, "window": 0, "sinks": 0},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["tables", "append", "append", "append4", "window", "window", "kv4", "kv4"])
        H_Q, H_KV = rng.choice(HEADS)
        page = rng.choice([32, 64, 96, 128, 256])
        if op == "tables":
            return {"op": op, "B": _log_int(rng, 1, 1024), "new": rng.choice(["one", "mixed", "prompts"]),
                    "page": rng.choice([16, page]), "lens": rng.choice(["uniform", "lognormal", "bimodal"]),
                    "len_lo": rng.choice([0, 1, 16]), "len_hi": _log_int(rng, 64, 32768),
                    "len_seed": rng.randrange(1 << 20), "pool": rng.choice([0.5, 0.95, 1.25])}
        if op in ("append", "append4"):
            case = {"op": op, "N": _log_int(rng, 1, 16384), "H_KV": H_KV, "page": page}
            if op == "append":
                case.update(H_Q=H_Q, rot=rng.choice([0, 32, 64, 96, 128]), pairs=rng.choice(["halves", "neighbours"]),
                            norm=rng.choice([True, True, False]), far=_log_int(rng, 1024, 131072))
            if case["N"] * (case.get("H_Q", 0) + 2 * H_KV) <= MAX_TOKEN_HEADS:
                return case
            continue
        case = {"op": op, "B": _log_int(rng, 1, 128), "H_Q": H_Q, "H_KV": H_KV, "page": page}
        hi = _log_int(rng, 40, 32768)
        case.update(lens=rng.choice(["uniform", "lognormal", "bimodal"]),
                    len_lo=rng.choice([0, 1, 16, max(1, hi // 16), hi]), len_hi=hi, len_seed=rng.randrange(1 << 20))
        if op == "window" or rng.random() < 0.3:
            case.update(window=_log_int(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 33, 128]))
        else:
            case.update(window=0, sinks=0)
        if op == "window":
            case["layout"] = rng.choice(["dense", "packed", "paged"])
            if case["layout"] == "dense":
                case["len_lo"] = hi
        lens = _lengths(case)
        row = H_KV * D * 4
        if 0 < sum(lens) * row <= MAX_KV_BYTES and len(lens) * max(lens) * row <= MAX_PADDED:
            return case


def _lengths(case):
    rng = np.random.default_rng(case["len_seed"])
    B, lo, hi = case["B"], case["len_lo"], case["len_hi"]
    if case["lens"] == "uniform":
        x = rng.integers(lo, hi + 1, B)
    elif case["lens"] == "lognormal":
        x = np.clip(rng.lognormal(math.log(max(lo, hi / 16, 1)), 1.0, B), lo, hi)
    else:  # bimodal: one sequence in eight at the full length, the others at a thirty-second of it
        x = np.where(rng.permutation(B) < max(1, B // 8), hi, max(lo, hi // 32))
    return [int(v) for v in x]


def _new_lengths(case):
    """Tokens each request brings: one, a prompt piece of up to 512, or a mixture with idle requests."""
    rng = np.random.default_rng(case["len_seed"] + 1)
    B = case["B"]
    if case["new"] == "one":
        return [1] * B
    piece = rng.integers(1, 513, B)
    if case["new"] == "prompts":
        return [int(v) for v in piece]
    kind = rng.integers(0, 8, B)
    return [int(v) for v in np.where(kind == 0, piece, np.where(kind == 1, 0, 1))]


def _visible(case, L):
    """Keys of a sequence of L that its query sees."""
    return L if not case["window"] else min(L, case["window"] + min(case["sinks"], L))


# ---------------------------------------------------------------- inputs


def _normal(g, shape, scale=1.0):
    x = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    return x.normal_(0.0, scale, generator=g)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _generators(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    cpu = torch.Generator()
    cpu.manual_seed(seed + 1)
    return g, cpu


def _tables_state(case, seed):
    _, cpu = _generators(seed)
    page, B = case["page"], case["B"]
    order = torch.randperm(B, generator=cpu).tolist()
    lens, new = _lengths(case), _new_lengths(case)
    lens, new = [lens[i] for i in order], [new[i] for i in order]
    held = [-(-n // page) for n in lens]
    need = [-(-(a + b) // page) - h for a, b, h in zip(lens, new, held)]
    num_free = max(1, int(sum(need) * case["pool"]))
    taken = 7
    ids = torch.randperm(sum(held) + taken + num_free, generator=cpu).to(torch.int32)
    table = torch.full((B, max(h + n for h, n in zip(held, need)) + 2), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = ids[at:at + n]
        at += n
    return {"lens": _ints(lens), "new": _ints(new), "free": ids[at:].contiguous().to(DEV), "taken": _ints([taken]),
            "table": table.to(DEV), "page": page, "num_pages": ids.numel(), "rows": sum(new) + 3}


def _slots(cpu, N, rows):
    """Distinct rows of a cache for N tokens, in runs as pages give them, in random order of runs."""
    runs = torch.randperm(rows // 32, generator=cpu)[: -(-N // 32)]
    return (runs[:, None] * 32 + torch.arange(32)).reshape(-1)[:N].to(torch.int32).to(DEV)


def _append_state(case, seed):
    g, cpu = _generators(seed)
    N, H_KV, page = case["N"], case["H_KV"], case["page"]
    pages = -(-N // page) + 2
    H_Q = case.get("H_Q", 0)
    # one projection's output: q, k and v of a token side by side, some channels far larger than others
    x = _normal(g, (N, H_Q + 2 * H_KV, D), 2.0)
    x[:, :, 5] *= 8.0
    s = {"slots": _slots(cpu, N, pages * page), "k": x[:, H_Q:H_Q + H_KV], "v": x[:, H_Q + H_KV:]}
    if case["op"] == "append4":
        s["cache"] = _packed(_normal(g, (pages, page, H_KV, D)), _normal(g, (pages, page, H_KV, D)))
        return s
    s["q"] = x[:, :H_Q]
    s["k_cache"] = _normal(g, (pages, page, H_KV, D))
    s["v_cache"] = _normal(g, (pages, page, H_KV, D))
    s["positions"] = torch.randint(0, case["far"], (N,), generator=g, dtype=torch.int32, device=DEV)
    s["wq"] = s["wk"] = s["rope"] = None
    if case["norm"]:
        s["wq"] = (1 + 0.25 * _normal(g, (D,)).float()).bfloat16()
        s["wk"] = (1 + 0.25 * _normal(g, (D,)).float()).bfloat16()
    if case["rot"]:
        half = case["rot"] // 2
        inv = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        angle = torch.arange(case["far"], dtype=torch.float64, device=DEV)[:, None] * inv
        s["rope"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    s["neighbours"] = case["pairs"] == "neighbours"
    return s


def _paging(cpu, lens, page):
    pages = [-(-n // page) for n in lens]
    num = sum(pages) + 8
    order = torch.randperm(num, generator=cpu).to(torch.int32)
    table = torch.zeros(len(lens), max(max(pages), 1), dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return num, table.to(DEV)


def _attention_state(case, seed):
    g, cpu = _generators(seed)
    B, H_Q, H_KV = case["B"], case["H_Q"], case["H_KV"]
    lens = _lengths(case)
    s = {"L": max(lens), "window": case["window"], "sinks": case["sinks"], "seq_lens": _ints(lens),
         "q": _normal(g, (B, H_Q, D), 2.0), "lse": torch.empty(B, H_Q, dtype=torch.float32, device=DEV)}
    layout = case.get("layout", "paged")
    if layout == "paged":
        num, s["table"] = _paging(cpu, lens, case["page"])
        shape = (num, case["page"], H_KV, D)
    elif layout == "packed":
        s["cu"] = _ints(np.concatenate([[0], np.cumsum(lens)]))
        shape = (sum(lens), H_KV, D)
    else:
        shape = (B, case["len_hi"], H_KV, D)
    if case["op"] == "kv4":
        s["cache"] = torch.empty(num, H_KV, case["page"] // TILE, TILE_BYTES, dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 17) // (case["page"] * H_KV))
        for i in range(0, num, step):  # a part at a time: the 32-bit values would take eight times the cache
            part = (min(step, num - i), case["page"], H_KV, D)
            s["cache"][i:i + step] = _packed(_normal(g, part), _normal(g, part))
    else:
        s["k"] = _normal(g, shape)
        s["v"] = _normal(g, shape)
    return s


def prepare(case, seed):
    state = _tables_state if case["op"] == "tables" else _append_state if "N" in case else _attention_state
    return {"op": case["op"], **state(case, seed)}


# ---------------------------------------------------------------- plain forms


def _codes(x):
    """4-bit codes [..., D] and scale bytes [..., D / 32] of float32 rows that hold bf16 values."""
    blocks = x.unflatten(-1, (D // 32, 32))
    _, e = torch.frexp(blocks.abs().amax(dim=-1) / 7)  # the least power of two that is no less: 2^e, or 2^(e - 1)
    m = blocks.abs().amax(dim=-1)
    e = torch.where(m <= 7 * torch.exp2((e - 1).float()), e - 1, e).clamp(-125, 125)
    y = blocks / torch.exp2(e.float())[..., None]
    a = y.abs()
    up = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    return (up + 8 * torch.signbit(y).int()).flatten(-2).to(torch.uint8), (e + 127).to(torch.uint8)


def _scale_places(slot_row):
    """Where a key's four K scales sit in its block's 256 scale bytes; [..., 4]."""
    g = torch.arange(4, device=slot_row.device)
    return 4 * (4 * (slot_row[..., None] % 16) + g) + slot_row[..., None] // 16


def _put(cache, slots, k, v):
    """Rows k, v float32 [N, H_KV, D] into the cache's rows `slots`."""
    num, H_KV, blocks, _ = cache.shape
    slots = slots.long()
    page, at = slots // (blocks * TILE), slots % (blocks * TILE)
    h = torch.arange(H_KV, device=DEV)
    start = ((page[:, None] * H_KV + h) * blocks + (at // TILE)[:, None]) * TILE_BYTES  # [N, H_KV]
    flat, row = cache.view(-1), (at % TILE)[:, None].expand(-1, H_KV)
    put = []
    ks, vs = _codes(k), _codes(v)
    for codes, first in ((ks[0], 0), (vs[0], TILE * 64)):
        put.append(((start + first + row * 64)[..., None] + torch.arange(64, device=DEV),
                    codes[..., 0::2] | codes[..., 1::2] << 4))
    for scales, first in ((ks[1], 0), (vs[1], 2)):
        put.append((start[..., None] + TILE * 128 + first + _scale_places(row), scales))
    for i, x in put:
        flat[i.reshape(-1)] = x.reshape(-1)


def _packed(k, v):
    """A cache of the bf16 rows [pages, page, H_KV, D]."""
    pages, page, H_KV, _ = k.shape
    cache = torch.empty(pages, H_KV, page // TILE, TILE_BYTES, dtype=torch.uint8, device=DEV)
    _put(cache, torch.arange(pages * page, device=DEV), k.reshape(-1, H_KV, D).float(), v.reshape(-1, H_KV, D).float())
    return cache


def _values(cache, page, at):
    """K and V float32 [..., H_KV, D] of the cache's rows `at` of pages `page` [...]."""
    pair = torch.arange(256, device=cache.device)
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=cache.device)
    of = torch.cat([mag, -mag])
    lut = torch.stack([of[pair % 16], of[pair // 16]], dim=1)
    block, r = at // TILE, at % TILE
    codes = cache[..., :TILE * 128].unflatten(-1, (2, TILE, 64))[page, :, block, :, r]  # [..., H_KV, 2, 64]
    x = torch.index_select(lut, 0, codes.reshape(-1).int()).view(*codes.shape[:-1], 4, 32)
    scales = cache[..., TILE * 128:].unflatten(-1, (16, 4, 2, 2))[page, :, block, r % 16, :, :, r // 16]
    scales = torch.exp2(scales.float() - 127.0).transpose(-1, -2)  # [..., H_KV, 2, 4]
    x = (x * scales[..., None]).flatten(-2)
    return x[..., 0, :], x[..., 1, :]


def _norm_rotate(x, w, rope, positions, neighbours):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w.float()
    if rope is None:
        return x
    half = rope.shape[1] // 2
    cs = rope[positions.long()]
    c, s = cs[:, None, :half], cs[:, None, half:]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if neighbours else (r[..., :half], r[..., half:])
    ra, rb = a * c - b * s, b * c + a * s
    r = torch.stack([ra, rb], dim=-1).flatten(-2) if neighbours else torch.cat([ra, rb], dim=-1)
    return torch.cat([r, rest], dim=-1)


def _plain_tables(s):
    lens, new, page, table = s["lens"].long(), s["new"].long(), s["page"], s["table"]
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    held = (lens + page - 1) // page
    fits = (lens + new <= table.shape[1] * page) & (cu[1:] <= s["rows"])
    need = torch.where(fits, (lens + new + page - 1) // page - held, 0)
    upto = need.cumsum(0)
    avail = s["free"].numel() - s["taken"].long()
    fits &= (need == 0) | (upto <= avail)
    need = torch.where(fits, need, 0)
    first = s["taken"].long() + upto - need
    j = torch.arange(table.shape[1], device=DEV)[None] - held[:, None]
    grown = torch.where((j >= 0) & (j < need[:, None]),
                        s["free"][(first[:, None] + j).clamp(0, s["free"].numel() - 1)], table)
    table.copy_(grown)
    row = torch.arange(s["rows"], device=DEV)
    b = torch.searchsorted(cu, row, right=True) - 1
    live = row < cu[-1]
    b = b.clamp(max=lens.numel() - 1)
    pos = torch.where(live, lens[b] + row - cu[b], 0)
    at = grown[b, (pos // page).clamp(max=table.shape[1] - 1)].long()
    slot = torch.where(live & fits[b], at * page + pos % page, -1)
    taken = s["taken"].long() + (need.cumsum(0))[-1]
    i32 = torch.int32
    return (table, torch.where(fits, lens + new, lens).to(i32), taken.to(i32), cu.to(i32), slot.to(i32), pos.to(i32))


def _attend(q, k, v, seen):
    """q [B, H_Q, D], k and v [B, V, H_KV, D] and which keys are seen [B, V]: out bf16, lse; a row that sees nothing
    gives zeros and -inf."""
    B, H_Q, _ = q.shape
    H_KV = k.shape[2]
    qg = q.float().view(B, H_KV, H_Q // H_KV, D)
    sc = torch.matmul(qg, k.float().permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    sc = sc.masked_fill(~seen[:, None, None, :], -math.inf)
    m = sc.amax(dim=-1, keepdim=True)
    p = torch.exp(sc - m.clamp(min=-3e38))
    l = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v.float().permute(0, 2, 1, 3).contiguous()) / l.clamp(min=1e-30)
    return o.reshape(B, H_Q, D).bfloat16(), (m + torch.log(l)).reshape(B, H_Q)


def _seen(s):
    """Positions [B, V] of the keys to look at, and which of them the query sees."""
    L = s["seq_lens"].long()[:, None]
    W, S = s["window"], s["sinks"]
    if not W or W + S >= s["L"]:
        j = torch.arange(max(s["L"], 1), device=DEV)[None].expand(L.shape[0], -1)
        return j, (j < L) & ((j < S) | (j >= L - W) if W else True)
    j = torch.arange(W + S, device=DEV)[None]
    pos = torch.where(j < S, j, L - W + j - S)  # the sinks, then the window
    seen = (pos >= 0) & (pos < L) & ((j < S) | (pos >= S))
    return pos.clamp(min=0).minimum((L - 1).clamp(min=0)), seen


def _plain_window(s):
    pos, seen = _seen(s)
    b = torch.arange(pos.shape[0], device=DEV)[:, None]
    if "table" in s:
        page = s["k"].shape[1]
        row = s["table"].long()[b, pos.clamp(max=s["table"].shape[1] * page - 1) // page] * page + pos % page
    elif "cu" in s:
        row = (s["cu"].long()[:-1, None] + pos).clamp(max=max(s["k"].shape[0] - 1, 0))
    else:
        row = b * s["k"].shape[1] + pos.clamp(max=s["k"].shape[1] - 1)
    k, v = (x.reshape(-1, *x.shape[-2:])[row] for x in (s["k"], s["v"]))
    return _attend(s["q"], k, v, seen)


def _plain_kv4(s):
    pos, seen = _seen(s)
    page = s["cache"].shape[2] * TILE
    b = torch.arange(pos.shape[0], device=DEV)[:, None]
    k, v = _values(s["cache"], s["table"].long()[b, (pos // page).clamp(max=s["table"].shape[1] - 1)], pos % page)
    return _attend(s["q"], k, v, seen)


def _plain(s):
    op = s["op"]
    if op == "tables":
        return _plain_tables(s)
    if op == "append":
        at = s["slots"].long()
        q = _norm_rotate(s["q"], s["wq"], s["rope"], s["positions"], s["neighbours"]).bfloat16()
        s["k_cache"].flatten(0, 1)[at] = _norm_rotate(s["k"], s["wk"], s["rope"], s["positions"],
                                                      s["neighbours"]).bfloat16()
        s["v_cache"].flatten(0, 1)[at] = s["v"]
        return q, s["k_cache"], s["v_cache"]
    if op == "append4":
        _put(s["cache"], s["slots"], s["k"].float(), s["v"].float())
        page = s["cache"].shape[2] * TILE
        row = torch.arange(s["cache"].shape[0] * page, device=DEV)
        return [x.bfloat16() for x in _values(s["cache"], row // page, row % page)]
    return _plain_window(s) if op == "window" else _plain_kv4(s)


def run(s):
    if not own:
        return _plain(s)
    import paper_2604_00028_amd as da
    op = s["op"]
    if op == "tables":
        lens, taken, cu, slots, positions = da.da_extend_tables(s["lens"], s["new"], s["free"], s["taken"], s["table"],
                                                                s["page"], s["num_pages"], s["rows"])
        return s["table"], lens, taken, cu, slots, positions
    if op == "append":
        q = da.da_append_kv(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["k_cache"], s["v_cache"],
                            rope=s["rope"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS, neighbours=s["neighbours"])
        return q, s["k_cache"], s["v_cache"]
    if op == "append4":
        da.da_append_kv4(None, s["k"], s["v"], None, s["slots"], s["cache"])
        return list(da.da_read_kv4(s["cache"]))
    if op == "window":
        out = da.da_decode_attn_window(s["q"], s["k"], s["v"], s["window"], s["sinks"], s.get("cu"), s.get("table"),
                                       s["seq_lens"] if "table" in s else None, L_K_max=s["L"], lse_out=s["lse"])
        return out, s["lse"]
    out = da.da_decode_attn_kv4(s["q"], s["cache"], s["table"], s["seq_lens"], s["L"], s["window"], s["sinks"],
                                lse_out=s["lse"])
    return out, s["lse"]


def work(case):
    op = case["op"]
    if op == "tables":
        B, page = case["B"], case["page"]
        lens, new = _lengths(case), _new_lengths(case)
        need = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(lens, new))
        return {"bytes": 4 * (4 * B + 3 + 2 * (sum(new) + 3) + 2 * need), "flops": sum(new) + 4 * B}
    if op == "append":
        heads = case["H_Q"] + 2 * case["H_KV"]
        return {"bytes": case["N"] * (heads * D * 4 + 8 + 4 * case["rot"]),
                "flops": case["N"] * (case["H_Q"] + case["H_KV"]) * D * 8}
    if op == "append4":
        pages = -(-case["N"] // case["page"]) + 2
        rows = case["N"] + pages * case["page"]  # written, and read back
        return {"bytes": rows * 2 * case["H_KV"] * (D * 2 + 68) + 4 * case["N"], "flops": rows * 2 * case["H_KV"] * D * 2}
    keys = sum(_visible(case, L) for L in _lengths(case))
    rows = case["B"] * case["H_Q"]
    per_key = case["H_KV"] * (136 if op == "kv4" else D * 4)
    return {"bytes": keys * per_key + rows * (D * 4 + 4), "flops": 4 * keys * case["H_Q"] * D}


# ---------------------------------------------------------------- the definitions in 64 bits


def _e2m1(code):
    """The value of 4-bit codes: sign, two exponent bits, one mantissa bit."""
    e, m = (code >> 1) & 3, code & 1
    mag = torch.where(e == 0, 0.5 * m.double(), torch.ldexp(1 + 0.5 * m.double(), e - 1))
    return torch.where(code >= 8, -mag, mag)


def _exact_rows(cache, rows):
    """K and V of the cache's rows (a list of row numbers): float64 [n, H_KV, D] each."""
    _, H_KV, blocks, _ = cache.shape
    rows = rows.long()
    tile = cache.permute(0, 2, 1, 3).reshape(-1, H_KV, TILE_BYTES)[rows // TILE]  # [n, H_KV, TILE_BYTES]
    r = rows % TILE
    n = torch.arange(rows.numel(), device=rows.device)
    d = torch.arange(D, device=rows.device)
    got = []
    for v in (0, 1):
        byte = tile[n[:, None], :, 2048 * v + r[:, None] * 64 + d // 2].permute(0, 2, 1).int()  # [n, H_KV, D]
        code = torch.where(d % 2 == 1, byte >> 4, byte & 15)
        place = 4096 + 4 * (4 * (r % 16)[:, None] + d // 32) + (r // 16)[:, None] + 2 * v
        e = tile[n[:, None], :, place].permute(0, 2, 1).int() - 127
        got.append(torch.ldexp(_e2m1(code), e))
    return got


def _exact_quantised(x):
    """What rows of bf16 values become in the 4-bit cache, by search over the values there are."""
    x = x.double().unflatten(-1, (4, 32))
    m = x.abs().amax(dim=-1, keepdim=True)
    powers = torch.ldexp(torch.ones(251, dtype=torch.float64, device=x.device), torch.arange(-125, 126, device=x.device))
    i = torch.searchsorted(7 * powers, m).clamp(max=250)
    scale = powers[i]
    a = x.abs() / scale
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    best = torch.zeros_like(a)
    for n in range(1, 8):  # the nearer one; a tie goes to the even code
        mid = (grid[n - 1] + grid[n]) / 2
        best = torch.where((a > mid) | ((a == mid) & (n % 2 == 0)), grid[n], best)
    return (torch.copysign(best, x) * scale).flatten(-2)


def _exact_append(s):
    at = s["slots"].long()

    def turned(x, w):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + EPS) * w.double()
        if s["rope"] is None:
            return y
        half = s["rope"].shape[1] // 2
        z = torch.complex(s["rope"][:, :half].double(), s["rope"][:, half:].double())[s["positions"].long()][:, None]
        i = torch.arange(half, device=y.device)
        i, j = (2 * i, 2 * i + 1) if s["neighbours"] else (i, i + half)
        p = torch.complex(y[..., i], y[..., j]) * z
        y = y.clone()
        y[..., i], y[..., j] = p.real, p.imag
        return y

    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    k_cache.flatten(0, 1)[at] = turned(s["k"], s["wk"])
    v_cache.flatten(0, 1)[at] = s["v"].double()
    return turned(s["q"], s["wq"]), k_cache, v_cache


def exact(case, seed):
    op = case["op"]
    if op == "tables":
        return None
    if op == "append":
        return _exact_append(_append_state(case, seed))
    if op == "append4":
        s = _append_state(case, seed)
        k, v = _exact_rows(s["cache"], torch.arange(s["cache"].shape[0] * case["page"], device=DEV))
        k[s["slots"].long()] = _exact_quantised(s["k"])
        v[s["slots"].long()] = _exact_quantised(s["v"])
        return [k, v]
    s = _attention_state(case, seed)
    lens, W, S = _lengths(case), case["window"], case["sinks"]
    H_Q, H_KV = case["H_Q"], case["H_KV"]
    outs, lses, at = [], [], 0
    for b, L in enumerate(lens):
        start, at = at, at + L
        j = torch.arange(L, device=DEV)
        if W:
            j = j[(j < S) | (j >= L - W)]
        if not L:
            outs.append(torch.zeros(H_Q, D, dtype=torch.float64, device=DEV))
            lses.append(torch.full((H_Q,), -math.inf, dtype=torch.float64, device=DEV))
            continue
        if "table" in s:
            rows = s["table"][b].long()[j // case["page"]] * case["page"] + j % case["page"]
        else:
            rows = j + (start if "cu" in s else b * case["len_hi"])
        if op == "kv4":
            k, v = _exact_rows(s["cache"], rows)
        else:
            k, v = (x.reshape(-1, H_KV, D)[rows].double() for x in (s["k"], s["v"]))
        q = s["q"][b].double().view(H_KV, -1, D)
        z = torch.matmul(q, k.permute(1, 2, 0).contiguous()) * D ** -0.5
        lse = torch.logsumexp(z, dim=-1, keepdim=True)
        outs.append(torch.matmul(torch.exp(z - lse), v.permute(1, 0, 2).contiguous()).reshape(H_Q, D))
        lses.append(lse.reshape(H_Q))
    return torch.stack(outs), torch.stack(lses)
