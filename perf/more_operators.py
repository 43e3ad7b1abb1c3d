"""A bounded cache shared by many requests, as cases that can be timed and
checked: attention of a batch whose sequences share a prompt, the weights its
keys received, eviction of the keys that received least, and rows with
positions on several axes on their way into the cache.

Each case is one `op` with its sizes:

  prefix   da_decode_attn_prefix: groups of sequences share their first keys, which are read once a group
  weights  da_add_key_weights: the attention weight of every key, summed over the heads that share it and over steps
  evict    da_evict_kv: sequences past a budget keep the keys of most weight; pages go back to the free list
  axes     da_append_kv_axes: norms, rotation by positions on several axes, rows into a bf16 cache
  axes4    da_append_kv4_axes: the same into a cache of 4-bit values, which da_read_kv4 reads back

With `own` false, run() computes the same in elementary torch operations in 32
bits.  Lengths and groups of a batch follow from the case alone, so its work is
known; the seed of prepare() draws the tensors and the order of pages.
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
MAX_BYTES = 7 * 10 ** 8    # of a drawn case: the largest listed ones take as much
MAX_FLOPS = 7 * 10 ** 10
MAX_PADDED = 4 << 30       # keys and values in 32 bits with every sequence padded to the longest


def listed():
    return [
        # two samples of one short prompt: bound by latency
        {"name": "prefix_b2_l500", "op": "prefix", "B": 2, "H_Q": 64, "H_KV": 8, "page": 64, "groups": 1,
         "pre_lo": 500, "pre_hi": 500, "lens": "uniform", "len_lo": 17, "len_hi": 40, "len_seed": 11},
        # several prompts of odd lengths with few requests each, own parts of mixed lengths
        {"name": "prefix_b24_g5", "op": "prefix", "B": 24, "H_Q": 32, "H_KV": 4, "page": 32, "groups": 5,
         "pre_lo": 100, "pre_hi": 6001, "lens": "lognormal", "len_lo": 1, "len_hi": 4000, "len_seed": 12},
        # a server's system prompt of 8192 tokens under 32 requests with short own parts
        {"name": "prefix_b32_p8192", "op": "prefix", "B": 32, "H_Q": 64, "H_KV": 8, "page": 64, "groups": 1,
         "pre_lo": 8192, "pre_hi": 8192, "lens": "uniform", "len_lo": 16, "len_hi": 512, "len_seed": 13},
        # the largest: 128 requests over one document of 16384 tokens
        {"name": "prefix_b128_p16384", "op": "prefix", "B": 128, "H_Q": 64, "H_KV": 8, "page": 64, "groups": 1,
         "pre_lo": 16384, "pre_hi": 16384, "lens": "uniform", "len_lo": 100, "len_hi": 1500, "len_seed": 14},
        # one context: the weights of 4001 keys
        {"name": "weights_b1_l4001", "op": "weights", "B": 1, "H_Q": 64, "H_KV": 8, "page": 64,
         "lens": "uniform", "len_lo": 4001, "len_hi": 4001, "len_seed": 1, "decay": 1.0},
        # a loaded server with a budget of 8192 keys, old weights fading
        {"name": "weights_b32_l8192", "op": "weights", "B": 32, "H_Q": 64, "H_KV": 8, "page": 64,
         "lens": "uniform", "len_lo": 8000, "len_hi": 8256, "len_seed": 21, "decay": 0.98},
        # every sequence of a decode batch one key past its budget, after many such steps
        {"name": "evict_step_b32", "op": "evict", "B": 32, "H_KV": 8, "page": 64, "lens": "uniform", "len_lo": 4097,
         "len_hi": 4097, "len_seed": 31, "budget": 4096, "sinks": 4, "recent": 256, "history": True},
        # after the prompts: long ones shrink to 2048 keys
        {"name": "evict_prompt_b8", "op": "evict", "B": 8, "H_KV": 8, "page": 64, "lens": "uniform", "len_lo": 5000,
         "len_hi": 16000, "len_seed": 32, "budget": 2048, "sinks": 16, "recent": 512, "history": False},
        # pure MQA, odd lengths on both sides of an odd budget, some requests idle
        {"name": "evict_mqa_b61", "op": "evict", "B": 61, "H_KV": 1, "page": 96, "lens": "uniform", "len_lo": 0,
         "len_hi": 2900, "len_seed": 33, "budget": 1001, "sinks": 0, "recent": 33, "history": True},
        # one decode token of Llama-3.1-70B's heads, three axes
        {"name": "axes_n1", "op": "axes", "N": 1, "H_Q": 64, "H_KV": 8, "page": 64, "rot": 128, "pairs": "halves",
         "norm": True, "axes": 3, "order": "sections", "far": 8192},
        # a prompt of images of 8192 tokens
        {"name": "axes_n8192", "op": "axes", "N": 8192, "H_Q": 64, "H_KV": 8, "page": 64, "rot": 128,
         "pairs": "halves", "norm": True, "axes": 3, "order": "sections", "far": 16384},
        # an image of odd size into the 4-bit cache, axes taking turns over neighbouring pairs
        {"name": "axes4_n1501", "op": "axes4", "N": 1501, "H_Q": 32, "H_KV": 4, "page": 32, "rot": 64,
         "pairs": "neighbours", "norm": True, "axes": 2, "order": "turns", "far": 4096},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["prefix", "prefix", "prefix", "weights", "weights", "evict", "evict", "axes", "axes4"])
        H_Q, H_KV = rng.choice(HEADS)
        page = rng.choice([32, 64, 96, 128, 256])
        if op in ("axes", "axes4"):
            case = {"op": op, "N": _log_int(rng, 1, 16384), "H_Q": H_Q, "H_KV": H_KV, "page": page,
                    "rot": rng.choice([32, 64, 96, 128]), "pairs": rng.choice(["halves", "neighbours"]),
                    "norm": rng.choice([True, True, False]), "axes": rng.choice([1, 2, 3, 3, 4]),
                    "order": rng.choice(["sections", "turns"]), "far": _log_int(rng, 1024, 131072)}
        else:
            case = {"op": op, "B": _log_int(rng, 1, 128), "H_KV": H_KV, "page": page,
                    "lens": rng.choice(["uniform", "lognormal", "bimodal"])}
            hi = _log_int(rng, 16, 4096 if op == "prefix" else 16384)
            case.update(len_lo=min(hi, rng.choice([0, 1, 16, max(1, hi // 16), hi])), len_hi=hi,
                        len_seed=rng.randrange(1 << 20))
            if op == "evict":
                budget = _log_int(rng, 8, hi)
                sinks = rng.choice([0, 1, 4, 33, budget // 4])
                case.update(budget=budget, sinks=min(sinks, budget // 2), recent=rng.randrange(budget // 2 + 1),
                            history=rng.choice([True, False]))
            else:
                case["H_Q"] = H_Q
            if op == "prefix":
                pre = _log_int(rng, 32, 16384)
                case.update(groups=min(case["B"], _log_int(rng, 1, 16)), pre_lo=rng.choice([0, pre // 8, pre]),
                            pre_hi=pre)
            if op == "weights":
                case["decay"] = rng.choice([0.0, 0.5, 0.98, 1.0])
            lens = _lengths(case)
            if max(lens) <= case.get("budget", 0) or len(lens) * max(lens) * H_KV * D * 8 > MAX_PADDED:
                continue
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
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


def _groups(case):
    """Sequences and prefix keys of each group."""
    rng = np.random.default_rng(case["len_seed"] + 1)
    B, G = case["B"], case["groups"]
    cuts = np.sort(rng.choice(np.arange(1, B), G - 1, replace=False)) if G > 1 else np.array([], dtype=int)
    sizes = np.diff(np.concatenate([[0], cuts, [B]]))
    return [int(n) for n in sizes], [int(n) for n in rng.integers(case["pre_lo"], case["pre_hi"] + 1, G)]


def work(case):
    op = case["op"]
    if op in ("axes", "axes4"):
        N, H_Q, H_KV = case["N"], case["H_Q"], case["H_KV"]
        row = 2 * D
        kept = 2 * N * H_KV * (row if op == "axes" else 68)
        read_back = 2 * N * H_KV * (68 + row) if op == "axes4" else 0
        table = N * case["rot"] * 4
        return {"bytes": N * (H_Q + 2 * H_KV) * row + N * H_Q * row + kept + read_back + table + 4 * N * (case["axes"] + 1),
                "flops": 8 * N * (H_Q + H_KV) * D}
    lens, H_KV = _lengths(case), case["H_KV"]
    if op == "evict":
        cut, over = case["budget"], [n for n in _lengths(case) if n > case["budget"]]
        # of a key and head: weight and position read and written; rows that move: those kept past the budget, at
        # least the recent ones there, and of the others the share that is kept
        moved = 0
        for n in over:
            late = n - cut
            sure = min(late, case["recent"])
            moved += sure + (late - sure) * max(0, cut - case["sinks"] - case["recent"]) // max(1, n)
        return {"bytes": H_KV * (16 * sum(lens) + 4 * D * 2 * moved), "flops": H_KV * sum(over)}
    B, H_Q = case["B"], case["H_Q"]
    if op == "weights":
        return {"bytes": H_KV * sum(lens) * (2 * D + 8) + B * H_Q * (2 * D + 4), "flops": 2 * D * H_Q * sum(lens)}
    sizes, pre = _groups(case)
    keys = sum(pre) + sum(lens)
    seen = sum(n * p for n, p in zip(sizes, pre)) + sum(lens)
    return {"bytes": 4 * D * H_KV * keys + B * H_Q * (4 * D + 4), "flops": 4 * D * H_Q * seen}


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


def _paging(cpu, lens, page, spare=8):
    pages = [-(-n // page) for n in lens]
    num = sum(pages) + spare
    order = torch.randperm(num, generator=cpu).to(torch.int32)
    table = torch.zeros(len(lens), max(max(pages), 1), dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return num, table, order


def _prefix_state(case, seed):
    g, cpu = _generators(seed)
    B, H_Q, H_KV, page = case["B"], case["H_Q"], case["H_KV"], case["page"]
    sizes, pre = _groups(case)
    cu = np.concatenate([[0], np.cumsum(sizes)])
    p_of = np.repeat(pre, sizes)
    lens = [int(a + b) for a, b in zip(p_of, _lengths(case))]
    # pages that the prefix fills are the group's; the page that it ends in is each sequence's own, with copies
    whole = [p // page for p in pre]
    own_pages = [-(-n // page) - int(p) // page for n, p in zip(lens, p_of)]
    num = sum(whole) + sum(own_pages) + 8
    order = torch.randperm(num, generator=cpu).to(torch.int32)
    table = torch.zeros(B, max(max(-(-n // page) for n in lens), 1), dtype=torch.int32)
    at = 0
    for i, (n, w) in enumerate(zip(sizes, whole)):
        table[cu[i]:cu[i + 1], :w] = order[at:at + w]
        at += w
        for b in range(cu[i], cu[i + 1]):
            table[b, w:w + own_pages[b]] = order[at:at + own_pages[b]]
            at += own_pages[b]
    k, v = _normal(g, (num, page, H_KV, D)), _normal(g, (num, page, H_KV, D))
    for i, (n, p) in enumerate(zip(sizes, pre)):
        rest = p % page
        if rest and n > 1:
            ids = table[cu[i]:cu[i + 1], p // page].long().to(DEV)
            for x in (k, v):
                x[ids, :rest] = x[ids[0], :rest].clone()
    return {"q": _normal(g, (B, H_Q, D), 2.0), "k": k, "v": v, "table": table.to(DEV), "lens": _ints(lens),
            "cu": _ints(cu), "pre": _ints(pre), "L": max(lens), "groups": list(zip(sizes, pre)), "host_lens": lens,
            "lse": torch.empty(B, H_Q, dtype=torch.float32, device=DEV)}


def _rows_of(table, page, b, n):
    """Cache rows of the first n keys of sequence b."""
    j = torch.arange(n, device=table.device)
    return table[b].long()[j // page] * page + j % page


def _weights_state(case, seed):
    g, cpu = _generators(seed)
    B, H_Q, H_KV, page = case["B"], case["H_Q"], case["H_KV"], case["page"]
    lens = _lengths(case)
    num, table, _ = _paging(cpu, lens, page)
    table = table.to(DEV)
    q, k = _normal(g, (B, H_Q, D), 2.0), _normal(g, (num, page, H_KV, D))
    lse = torch.full((B, H_Q), -math.inf, dtype=torch.float32, device=DEV)
    for b, n in enumerate(lens):  # as the attention of the step left it
        if n:
            kb = k.view(-1, H_KV, D)[_rows_of(table, page, b, n)].float().permute(1, 2, 0).contiguous()
            sc = torch.matmul(q[b].float().view(H_KV, -1, D), kb) / math.sqrt(D)
            lse[b] = torch.logsumexp(sc, dim=-1).reshape(-1)
    stride = max(lens) + 5
    w = torch.empty(B, H_KV, stride, device=DEV).exponential_(4.0, generator=g)
    return {"q": q, "k": k, "table": table, "lens": _ints(lens), "L": max(lens), "lse": lse, "weights": w,
            "sum": w.clone(), "decay": case["decay"], "host_lens": lens}


def _evict_state(case, seed):
    g, cpu = _generators(seed)
    B, H_KV, page, budget = case["B"], case["H_KV"], case["page"], case["budget"]
    lens = _lengths(case)
    num, table, ids = _paging(cpu, lens, page)
    held = sum(-(-n // page) for n in lens)
    stride = max(lens) + 3
    # sums of attention weights: a few keys hold most, many hold the same little or nothing
    w = torch.empty(B, H_KV, stride, device=DEV).normal_(generator=g).mul_(2.0).exp_()
    w = torch.where(w < 0.5, torch.floor(w * 8) / 8, w)
    L = _ints(lens)
    pos = torch.full((B, H_KV, stride), -1, dtype=torch.int32, device=DEV)
    totals = L.clone()
    if case["history"]:
        # rows of earlier evictions lie in no order behind the sinks; later rows stand where they were appended
        gone = torch.randint(1, 5000, (B,), generator=g, device=DEV, dtype=torch.int32)
        totals = torch.where(L >= budget, L + gone, L)
        settled = min(budget, stride)
        order = torch.rand(B, H_KV, max(settled - case["sinks"], 0), generator=g, device=DEV).argsort(dim=-1)
        pos[:, :, :settled] = torch.arange(settled, device=DEV, dtype=torch.int32)
        span = (totals - (L - settled) - case["sinks"]).clamp(min=1)  # positions the settled rows may have
        pos[:, :, case["sinks"]:settled] = (case["sinks"] + (order.double() + 1) / max(order.shape[-1], 1)
                                            * span[:, None, None] - 1).int()
        pos[L < budget] = -1
    return {"k": _normal(g, (num, page, H_KV, D)), "v": _normal(g, (num, page, H_KV, D)), "table": table.to(DEV),
            "lens": L, "totals": totals, "weights": w, "positions": pos, "free": ids.to(DEV), "taken": _ints([held]),
            "lens_out": torch.empty_like(L), "weights_out": w.clone(), "positions_out": pos.clone(),
            "taken_out": _ints([0]), "L": max(lens), "budget": budget, "sinks": case["sinks"], "recent": case["recent"]}


def _axis_of_pair(case):
    pairs, A = case["rot"] // 2, case["axes"]
    if case["order"] == "turns":
        return [i % A for i in range(pairs)]
    first = pairs // (A + 1)  # the first axis (time) has the smallest share
    rest = [(pairs - first) * i // max(A - 1, 1) for i in range(A)]
    return [0] * (first if A > 1 else pairs) + [a for a in range(1, A) for _ in range(rest[a] - rest[a - 1])]


def _axes_state(case, seed):
    g, cpu = _generators(seed)
    N, H_Q, H_KV, page, A = case["N"], case["H_Q"], case["H_KV"], case["page"], case["axes"]
    pages = -(-N // page) + 2
    # one projection's output: q, k and v of a token side by side, some channels far larger than others
    x = _normal(g, (N, H_Q + 2 * H_KV, D), 2.0)
    x[:, :, 5] *= 8.0
    runs = torch.randperm(pages * page // 32, generator=cpu)[: -(-N // 32)]
    slots = (runs[:, None] * 32 + torch.arange(32)).reshape(-1)[:N].to(torch.int32)
    # images of 24 x 36 patches after each other: the first axis counts images, the next two rows and columns
    t = torch.arange(N)
    start = int(torch.randint(0, case["far"] - 512, (1,), generator=cpu))
    steps = [t // 864, t % 864 // 36, t % 36, t]
    positions = torch.stack([(start + s) % case["far"] for s in steps[:A]])
    half = case["rot"] // 2
    inv = 500000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
    angle = torch.arange(case["far"], dtype=torch.float64, device=DEV)[:, None] * inv
    s = {"q": x[:, :H_Q], "k": x[:, H_Q:H_Q + H_KV], "v": x[:, H_Q + H_KV:], "slots": slots.to(DEV),
         "positions": positions.to(torch.int32).to(DEV), "rope": torch.cat([angle.cos(), angle.sin()], dim=1).float(),
         "axes": bytes(_axis_of_pair(case)), "neighbours": case["pairs"] == "neighbours", "wq": None, "wk": None}
    if case["norm"]:
        s["wq"] = (1 + 0.25 * _normal(g, (D,)).float()).bfloat16()
        s["wk"] = (1 + 0.25 * _normal(g, (D,)).float()).bfloat16()
    s["k_cache"], s["v_cache"] = _normal(g, (pages, page, H_KV, D)), _normal(g, (pages, page, H_KV, D))
    if case["op"] == "axes4":  # only the new tokens' rows are read back
        s["cache"] = torch.zeros(pages, H_KV, page // TILE, TILE_BYTES, dtype=torch.uint8, device=DEV)
        del s["k_cache"], s["v_cache"]
    return s


def prepare(case, seed):
    make = {"prefix": _prefix_state, "weights": _weights_state, "evict": _evict_state}.get(case["op"], _axes_state)
    return {"op": case["op"], **make(case, seed)}


# ---------------------------------------------------------------- plain forms


def _plain_prefix(s):
    B, H_Q, _ = s["q"].shape
    page, H_KV = s["k"].shape[1:3]
    kf, vf = s["k"].view(-1, H_KV, D), s["v"].view(-1, H_KV, D)
    out = torch.zeros(B, H_Q, D, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(B, H_Q, device=DEV)
    b0 = 0
    for n, p in s["groups"]:
        b1 = b0 + n
        qs = s["q"][b0:b1].float().view(n, H_KV, -1, D) / math.sqrt(D)
        g = qs.shape[2]
        # every row of the group against the shared keys
        rows = _rows_of(s["table"], page, b0, p)
        kp, vp = kf[rows].float(), vf[rows].float()
        qp = qs.permute(1, 0, 2, 3).reshape(H_KV, n * g, D)
        sp = torch.matmul(qp, kp.permute(1, 2, 0).contiguous()).view(H_KV, n, g, p).transpose(0, 1)
        # and each sequence's against its own
        most = max(max(s["host_lens"][b0:b1]) - p, 1)
        j = p + torch.arange(most, device=DEV)
        seen = j < s["lens"][b0:b1, None]
        at = (s["table"][b0:b1].long()[:, (j // page).clamp(max=s["table"].shape[1] - 1)] * page + j % page)
        ks, vs = kf[at].float(), vf[at].float()  # [n, most, H_KV, D]
        so = torch.matmul(qs, ks.permute(0, 2, 3, 1).contiguous()).masked_fill(~seen[:, None, None, :], -math.inf)
        sc = torch.cat([sp, so], dim=-1)
        m = sc.amax(dim=-1, keepdim=True)
        e = torch.exp(sc - m.clamp(min=-3e38))
        l = e.sum(dim=-1, keepdim=True)
        ep = e[..., :p].transpose(0, 1).reshape(H_KV, n * g, p)
        o = torch.matmul(ep, vp.transpose(0, 1).contiguous()).view(H_KV, n, g, D).transpose(0, 1)
        o = (o + torch.matmul(e[..., p:], vs.transpose(1, 2).contiguous())) / l.clamp(min=1e-30)
        out[b0:b1] = o.reshape(n, H_Q, D).bfloat16()
        lse[b0:b1] = (m + torch.log(l)).reshape(n, H_Q)
        b0 = b1
    return out, lse


def _plain_weights(s):
    B, H_Q, _ = s["q"].shape
    page, H_KV = s["k"].shape[1:3]
    j = torch.arange(max(s["L"], 1), device=DEV)
    at = s["table"].long()[:, (j // page).clamp(max=s["table"].shape[1] - 1)] * page + j % page
    k = s["k"].view(-1, H_KV, D)[at].float()  # [B, L, H_KV, D]
    sc = torch.matmul(s["q"].float().view(B, H_KV, -1, D), k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(D)
    add = torch.exp(sc - s["lse"].view(B, H_KV, -1, 1)).sum(dim=2)
    seen = (j < s["lens"][:, None])[:, None]
    old = s["weights"][..., : j.numel()]
    s["sum"][..., : j.numel()] = torch.where(seen, s["decay"] * old + add, s["sum"][..., : j.numel()])
    return s["sum"]


def _plain_evict(s):
    B, H_KV, stride = s["weights"].shape
    page, budget = s["k"].shape[1], s["budget"]
    L = s["lens"].long()[:, None, None]
    r = torch.arange(stride, device=DEV)
    shift = (s["totals"].long() - s["lens"].long())[:, None, None]
    pos = torch.where(s["positions"] >= 0, s["positions"].long(), r + shift)
    kept_all = (pos < s["sinks"]) | (pos >= s["totals"].long()[:, None, None] - s["recent"])
    key = torch.where(kept_all, math.inf, s["weights"].double())
    key = torch.where(r < L, key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, order, True) & (r < L)
    over = L > budget
    hole = ~kept & (r < budget) & over
    mover = kept & (r >= budget) & over
    b, h, dst = hole.nonzero(as_tuple=True)  # both in order of sequence, head and row, as many of each
    _, _, src = mover.nonzero(as_tuple=True)
    table = s["table"].long()
    to, of = (table[b, x // page] * page + x % page for x in (dst, src))
    for c in (s["k"], s["v"]):
        flat = c.view(-1, H_KV, D)
        flat[to, h] = flat[of, h]
    gone = over & (r >= budget)
    w, p = s["weights"].clone(), torch.where(over, pos, s["positions"].long())
    w[b, h, dst], p[b, h, dst] = s["weights"][b, h, src], pos[b, h, src]
    w, p = torch.where(gone, 0.0, w), torch.where(gone, -1, p)
    s["weights_out"].copy_(torch.where(r < L, w, s["weights_out"]))
    s["positions_out"].copy_(torch.where(r < L, p.int(), s["positions_out"]))
    # pages past the budget, in order of sequence, in front of the free ones
    i = torch.arange(table.shape[1], device=DEV)
    held = (s["lens"].long() + page - 1) // page
    free = (i >= -(-budget // page)) & (i < held[:, None]) & (s["lens"] > budget)[:, None]
    ids = table[free].int()
    first = s["taken"].long() - ids.numel()
    s["free"][first + torch.arange(ids.numel(), device=DEV)] = ids
    s["taken_out"].copy_(first)
    s["lens_out"].copy_(s["lens"].clamp(max=budget))
    return (s["lens_out"], s["weights_out"], s["positions_out"], s["taken_out"], s["free"], s["k"], s["v"])


def _rotate(x, w, s):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w.float()
    half = s["rope"].shape[1] // 2
    pair = torch.arange(half, device=DEV)
    at = s["positions"].long()[torch.tensor(list(s["axes"]), device=DEV)].t()  # [N, pairs]
    c, sn = (s["rope"][at, pair + i * half][:, None, :] for i in (0, 1))
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if s["neighbours"] else (r[..., :half], r[..., half:])
    ra, rb = a * c - b * sn, b * c + a * sn
    r = torch.stack([ra, rb], dim=-1).flatten(-2) if s["neighbours"] else torch.cat([ra, rb], dim=-1)
    return torch.cat([r, rest], dim=-1).bfloat16()


def _four_bits(x):
    """The values that 4 bits and a power of two for 32 of them leave of bf16 rows."""
    y = x.float().unflatten(-1, (D // 32, 32))
    m = y.abs().amax(dim=-1, keepdim=True)
    _, e = torch.frexp(m / 7)  # the least power of two that is no less: 2^e, or 2^(e - 1)
    e = torch.where(m <= 7 * torch.exp2((e - 1).float()), e - 1, e).clamp(-125, 125)
    scale = torch.exp2(e.float())
    a = (y / scale).abs()
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device)
    up = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    return (torch.copysign(mag[up.long()], y) * scale).flatten(-2).bfloat16()


def _plain_axes(s):
    q, k = _rotate(s["q"], s["wq"], s), _rotate(s["k"], s["wk"], s)
    if s["op"] == "axes4":
        return q, _four_bits(k), _four_bits(s["v"])
    slots = s["slots"].long()
    s["k_cache"].view(-1, *k.shape[1:])[slots] = k
    s["v_cache"].view(-1, *k.shape[1:])[slots] = s["v"]
    return q, s["k_cache"], s["v_cache"]


# ---------------------------------------------------------------- the library's


def _own(s):
    import paper_2604_00028_amd as da

    op = s["op"]
    if op == "prefix":
        out = da.da_decode_attn_prefix(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], s["pre"], s["L"],
                                       lse_out=s["lse"])
        return out, s["lse"]
    if op == "weights":
        return da.da_add_key_weights(s["q"], s["k"], s["table"], s["lens"], s["lse"], s["weights"], s["L"],
                                     decay=s["decay"], weights_out=s["sum"])
    if op == "evict":
        lens, w, pos, taken = da.da_evict_kv(
            s["k"], s["v"], s["table"], s["lens"], s["totals"], s["weights"], s["positions"], s["budget"], s["L"],
            sinks=s["sinks"], recent=s["recent"], free_pages=s["free"], taken=s["taken"], lens_out=s["lens_out"],
            weights_out=s["weights_out"], positions_out=s["positions_out"], taken_out=s["taken_out"])
        return lens, w, pos, taken, s["free"], s["k"], s["v"]
    kw = dict(rope=s["rope"], axes=s["axes"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS, neighbours=s["neighbours"])
    if op == "axes4":
        q = da.da_append_kv4_axes(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["cache"], **kw)
        return (q, *da.da_read_kv4(s["cache"], s["slots"]))
    q = da.da_append_kv_axes(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["k_cache"], s["v_cache"], **kw)
    return q, s["k_cache"], s["v_cache"]


def run(state):
    if own:
        return _own(state)
    plain = {"prefix": _plain_prefix, "weights": _plain_weights, "evict": _plain_evict}.get(state["op"], _plain_axes)
    return plain(state)


# ---------------------------------------------------------------- the definitions, in 64 bits


def _exact_prefix(case, s):
    B, H_Q, _ = s["q"].shape
    page, H_KV = s["k"].shape[1:3]
    out = torch.zeros(B, H_Q, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, H_Q), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["lens"].tolist()):
        if not n:
            continue
        rows = _rows_of(s["table"], page, b, n)
        for h in range(H_KV):
            group = slice(h * (H_Q // H_KV), (h + 1) * (H_Q // H_KV))
            k, v = (x.view(-1, H_KV, D)[rows, h].double() for x in (s["k"], s["v"]))
            sc = s["q"][b, group].double() @ k.t() / math.sqrt(D)
            lse[b, group] = torch.logsumexp(sc, dim=-1)
            out[b, group] = torch.exp(sc - lse[b, group, None]) @ v
    return out, lse


def _exact_weights(case, s):
    H_Q, H_KV = case["H_Q"], case["H_KV"]
    out = s["sum"].double()
    for b, n in enumerate(s["lens"].tolist()):
        rows = _rows_of(s["table"], case["page"], b, n)
        for h in range(H_KV if n else 0):
            group = slice(h * (H_Q // H_KV), (h + 1) * (H_Q // H_KV))
            sc = s["k"].view(-1, H_KV, D)[rows, h].double() @ s["q"][b, group].double().t() / math.sqrt(D)
            out[b, h, :n] = (case["decay"] * s["weights"][b, h, :n].double()
                             + torch.exp(sc - s["lse"][b, group].double()).sum(dim=1))
    return out


def _exact_evict(case, s):
    budget, page, H_KV = case["budget"], case["page"], case["H_KV"]
    w_in, p_in, table = s["weights"].cpu().numpy(), s["positions"].cpu().numpy(), s["table"].cpu().numpy()
    lens, totals = s["lens"].tolist(), s["totals"].tolist()
    w, p = s["weights_out"].double().cpu().numpy(), s["positions_out"].cpu().numpy()
    moves, back = [], []
    for b, L in enumerate(lens):
        w[b, :, :L], p[b, :, :L] = w_in[b, :, :L], p_in[b, :, :L]
        if L <= budget:
            continue
        back += table[b, -(-budget // page):-(-L // page)].tolist()
        for h in range(H_KV):
            pos = np.where(p_in[b, h, :L] >= 0, p_in[b, h, :L], np.arange(L) + totals[b] - L)
            safe = (pos < case["sinks"]) | (pos >= totals[b] - case["recent"])
            rank = np.lexsort((np.arange(L), -w_in[b, h, :L].astype(np.float64), ~safe))
            keep = np.sort(rank[:budget])
            holes = np.setdiff1d(np.arange(budget), keep)
            late = keep[keep >= budget]
            p[b, h, :L] = pos
            w[b, h, holes], p[b, h, holes] = w_in[b, h, late], pos[late]
            w[b, h, budget:L], p[b, h, budget:L] = 0.0, -1
            moves += [(table[b, d // page] * page + d % page, table[b, a // page] * page + a % page, h)
                      for d, a in zip(holes.tolist(), late.tolist())]
    taken = int(s["taken"]) - len(back)
    free = s["free"].clone()
    free[taken:taken + len(back)] = _ints(back)
    caches = []
    to, of, h = torch.tensor(moves, dtype=torch.int64, device=DEV).view(-1, 3).unbind(1)
    for x in (s["k"], s["v"]):
        y = x.clone()
        y.view(-1, H_KV, D)[to, h] = x.view(-1, H_KV, D)[of, h]
        caches.append(y.double())
    return (s["lens"].clamp(max=budget), torch.from_numpy(w).to(DEV), torch.from_numpy(p).to(DEV), _ints([taken]), free,
            *caches)


def _exact_axes(case, s):
    A = list(s["axes"])
    half = len(A)
    turned = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().mean(dim=-1, keepdim=True) + EPS) * w.double()
        y = x.clone()
        for i, axis in enumerate(A):
            cs = s["rope"][s["positions"][axis].long()].double()
            c, sn = cs[:, None, i], cs[:, None, half + i]
            a, b = (2 * i, 2 * i + 1) if case["pairs"] == "neighbours" else (i, i + half)
            y[..., a], y[..., b] = x[..., a] * c - x[..., b] * sn, x[..., b] * c + x[..., a] * sn
        turned.append(y)
    if case["op"] == "axes4":
        return turned[0], None, None  # a key next to a border of the 4-bit codes has two right values
    caches = []
    for x, y in ((s["k_cache"], turned[1]), (s["v_cache"], s["v"].double())):
        x = x.double()
        x.view(-1, *y.shape[1:])[s["slots"].long()] = y
        caches.append(x)
    return (turned[0], *caches)


def exact(case, seed):
    define = {"prefix": _exact_prefix, "weights": _exact_weights, "evict": _exact_evict}.get(case["op"], _exact_axes)
    return define(case, prepare(case, seed))
