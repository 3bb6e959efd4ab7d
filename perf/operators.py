"""The operators of the 4-bit paged cache: what they compute, in plain form and through this library, over the sizes they serve.

A service that keeps many requests decoding at once holds their final caches in pages, and in 4 bits per number:

  pages   request lengths change (a token each, a prompt that arrives, a request that ends): pages are taken from and given
          back to a pool, the block table follows, and every new row gets its slot (cf_pages_resize)
  rows    rows of keys and values go to their slots in 4 bits (cf_kv4_write), and come back as numbers (cf_kv4_read)
  attn    query rows attend a request's pages (cf_kv4_attn): a token each, or a few tokens under the causal mask

The cache's format.  A row of a kv head is cut into groups of 32 numbers.  A group has a bf16 scale, its largest magnitude
over 6 rounded to nearest even; each number is the scale times the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (ties to
the even code, larger values to 6).  A scale below 2^-126 is stored as 0, a group with a number that is not finite has a NaN as
its scale and zero codes.  A slot is page * page_rows + row.  A layer of the pool is [n_pages][kv_heads][page_rows / 16] blocks
of 18 * head_dim bytes, each with 16 rows: codes of the keys, codes of the values, scales of the keys, scales of the values;
`_split` says where a number's code lies.

Lengths are spread evenly over a case's range, their order differs from seed to seed.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------------- cases

def listed() -> List[Dict]:
    return [
        # a decoding step of a small batch: one more row for each request
        {"name": "pages_step", "kind": "pages", "requests": 16, "page_rows": 64, "cols": 64, "rows_lo": 1, "rows_hi": 2764,
         "grow_lo": 1, "grow_hi": 1, "new": 0, "gone": 0, "max_new": 1},
        # a busy service between two steps: most requests go on, some have ended, some arrive with prompts of their own
        {"name": "pages_mixed", "kind": "pages", "requests": 1021, "page_rows": 32, "cols": 160, "rows_lo": 0, "rows_hi": 4001,
         "grow_lo": 1, "grow_hi": 1, "new": 100, "gone": 90, "max_new": 1100},
        # a large batch of final caches, all at once
        {"name": "pages_fill", "kind": "pages", "requests": 256, "page_rows": 16, "cols": 512, "rows_lo": 0, "rows_hi": 0,
         "grow_lo": 0, "grow_hi": 8191, "new": 0, "gone": 0, "max_new": 8192},
        # the new token's rows of eight requests, one layer of a running model
        {"name": "rows_token", "kind": "rows", "dtype": "bf16", "kv_heads": 4, "head_dim": 128, "layers": 1, "requests": 8,
         "page_rows": 64, "cap": 1, "rows_lo": 1, "rows_hi": 1, "start_lo": 200, "start_hi": 3000, "pad": 0},
        # odd lengths and a padded row of a model with narrow heads, in fp32
        {"name": "rows_ragged_f32", "kind": "rows", "dtype": "f32", "kv_heads": 8, "head_dim": 64, "layers": 3, "requests": 5,
         "page_rows": 48, "cap": 391, "rows_lo": 0, "rows_hi": 391, "start_lo": 0, "start_hi": 100, "pad": 64},
        # final caches of a batch of multi-head requests after pruning, several layers in one call
        {"name": "rows_final", "kind": "rows", "dtype": "bf16", "kv_heads": 32, "head_dim": 128, "layers": 4, "requests": 8,
         "page_rows": 64, "cap": 2764, "rows_lo": 2000, "rows_hi": 2764, "start_lo": 0, "start_hi": 0, "pad": 0},
        # a toy model in fp32, requests of few rows or none
        {"name": "attn_tiny_f32", "kind": "attn", "dtype": "f32", "q_heads": 4, "kv_heads": 4, "head_dim": 64, "layers": 1,
         "requests": 5, "page_rows": 16, "rows_lo": 0, "rows_hi": 83, "q_len": 1},
        # a generated token for one request after pruning, one layer of a running model
        {"name": "attn_one_gqa", "kind": "attn", "dtype": "bf16", "q_heads": 12, "kv_heads": 2, "head_dim": 128, "layers": 1,
         "requests": 1, "page_rows": 64, "rows_lo": 1011, "rows_hi": 1011, "q_len": 1},
        # a generated token for a busy service of grouped-query requests of every length
        {"name": "attn_service_gqa", "kind": "attn", "dtype": "bf16", "q_heads": 28, "kv_heads": 4, "head_dim": 128, "layers": 1,
         "requests": 96, "page_rows": 32, "rows_lo": 17, "rows_hi": 6001, "q_len": 1},
        # stored queries of several layers over ragged caches, replayed in one call
        {"name": "attn_replay_layers", "kind": "attn", "dtype": "bf16", "q_heads": 32, "kv_heads": 8, "head_dim": 128,
         "layers": 4, "requests": 3, "page_rows": 48, "rows_lo": 333, "rows_hi": 4444, "q_len": 1},
        # a short follow-up question over the caches of four requests
        {"name": "attn_follow_up", "kind": "attn", "dtype": "bf16", "q_heads": 28, "kv_heads": 4, "head_dim": 128, "layers": 1,
         "requests": 4, "page_rows": 64, "rows_lo": 4000, "rows_hi": 16000, "q_len": 24},
        # a generated token for eight requests with every passage kept, multi-head
        {"name": "attn_long_mha", "kind": "attn", "dtype": "bf16", "q_heads": 32, "kv_heads": 32, "head_dim": 128, "layers": 1,
         "requests": 8, "page_rows": 64, "rows_lo": 19000, "rows_hi": 21600, "q_len": 1},
    ]


def _between(rng: random.Random, lo: int, hi: int) -> int:
    """An integer of [lo, hi], its logarithm uniform."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng: random.Random) -> Dict:
    kind = rng.choice(["pages", "rows", "attn", "attn"])
    page_rows = 16 * rng.choice([1, 1, 2, 2, 3, 4, 4, 5, 8, 16])
    if kind == "pages":
        requests, fresh = _between(rng, 1, 1024), rng.random() < 0.4
        rows_hi = 0 if fresh else _between(rng, 1, 4096)
        grow_hi = _between(rng, 1, 8192 if fresh else 64)
        if fresh:
            requests = min(requests, max(1, 2000000 // grow_hi))
        new = 0 if fresh else rng.randrange(0, requests // 8 + 1)
        gone = 0 if fresh else rng.randrange(0, requests // 8 + 1)
        max_new = max(grow_hi, _between(rng, 1, 1024) if new else 1)
        cols = -(-(max(rows_hi, max_new) + grow_hi) // page_rows) + rng.randrange(0, 9)
        return {"kind": kind, "requests": requests, "page_rows": page_rows, "cols": cols, "rows_lo": 0 if fresh else rng.randrange(0, rows_hi + 1),
                "rows_hi": rows_hi, "grow_lo": rng.randrange(0, grow_hi + 1), "grow_hi": grow_hi, "new": new, "gone": gone, "max_new": max_new}
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    q_heads, kv_heads, head_dim = rng.choice([(12, 2, 128), (28, 4, 128), (32, 8, 128), (32, 32, 128), (64, 4, 128), (4, 4, 64), (8, 2, 64), (16, 1, 128)])
    requests, layers = _between(rng, 1, 128), rng.choice([1, 1, 1, 2, 3, 4])
    row_bytes = kv_heads * head_dim * 2 * (2 if dtype == "bf16" else 4)
    if kind == "rows":
        most = max(1, 300000000 // (row_bytes * layers * requests))
        cap = 1 if rng.random() < 0.3 else _between(rng, 1, min(6000, most))
        lo = rng.randrange(0, cap + 1)
        start_hi = rng.randrange(0, 300)
        return {"kind": kind, "dtype": dtype, "kv_heads": kv_heads, "head_dim": head_dim, "layers": layers, "requests": requests,
                "page_rows": page_rows, "cap": cap, "rows_lo": lo, "rows_hi": cap, "start_lo": rng.randrange(0, start_hi + 1),
                "start_hi": start_hi, "pad": rng.choice([0, 0, 8, 64])}
    q_len = 1 if rng.random() < 0.6 else _between(rng, 2, 32)
    most = max(16, int(4.0e8 / (kv_heads * head_dim * layers * requests * max(1.0, q_len * q_heads / kv_heads / 16))))
    rows_hi = _between(rng, 1, min(24000, most))
    return {"kind": kind, "dtype": dtype, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "layers": layers,
            "requests": requests, "page_rows": page_rows, "rows_lo": rng.randrange(0, rows_hi + 1), "rows_hi": rows_hi, "q_len": q_len}


# ------------------------------------------------------------------------------------------------------ inputs

def _spread(lo: int, hi: int, n: int) -> np.ndarray:
    """n lengths from lo to hi, evenly."""
    return np.array([lo + (hi - lo) * i // max(1, n - 1) for i in range(n)], np.int64) if n > 1 else np.array([hi], np.int64)


def _spread_in_turn(lo: int, hi: int, n: int, seed: int) -> np.ndarray:
    return np.random.RandomState(seed % (1 << 31)).permutation(_spread(lo, hi, n))


def _targets(case: Dict):
    """(rows, rows after) of a "pages" case by rank: the last ones have ended, the ones before them arrive."""
    n, new, gone = case["requests"], case["new"], case["gone"]
    before = _spread(case["rows_lo"], case["rows_hi"], n)
    after = before + _spread(case["grow_lo"], case["grow_hi"], n)[::-1]
    if gone:
        after[n - gone:] = -1
    if new:
        before[n - gone - new:n - gone] = 0
        after[n - gone - new:n - gone] = _spread(1, case["max_new"], new)
    return before, after


def _random_pages(lengths: np.ndarray, page_rows: int, cols: int, spare: int, seed: int):
    """(table [B, cols] with -1 where a request has no page, the free pages as a stack, number of pages)."""
    need = -(-np.maximum(lengths, 0) // page_rows)
    n_pages = int(need.sum()) + spare
    order = np.random.RandomState((seed + 1) % (1 << 31)).permutation(n_pages).astype(np.int32)
    table = np.full((len(lengths), cols), -1, np.int32)
    has = np.arange(cols)[None, :] < need[:, None]
    table[has] = order[:int(need.sum())]
    return table, order[int(need.sum()):], n_pages


def _normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def prepare(case: Dict, seed: int) -> Dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return {"pages": _prepare_pages, "rows": _prepare_rows, "attn": _prepare_attn}[case["kind"]](case, seed, g)


def _page_state(table, rows, free, n_pages: int):
    """Table, lengths, free stack, its height and the status word, one after another in one buffer."""
    b, cols = table.shape
    stack = np.zeros(n_pages, np.int32)
    stack[:len(free)] = free
    flat = np.concatenate([table.reshape(-1), rows.astype(np.int32), stack, np.array([len(free), 0], np.int32)])
    return torch.from_numpy(flat).cuda()


def _views(case: Dict, flat: torch.Tensor, n_pages: int):
    b, cols = case["requests"], case["cols"]
    at = [0, b * cols, b * cols + b, b * cols + b + n_pages, b * cols + b + n_pages + 1, flat.numel()]
    table, rows, free, count, status = (flat[i:j] for i, j in zip(at, at[1:]))
    return table.view(b, cols), rows, free, count, status


def _prepare_pages(case, seed, g):
    before, after = _targets(case)
    order = np.random.RandomState(seed % (1 << 31)).permutation(len(before))
    before, after = before[order], after[order]
    need = -(-np.maximum(after, 0) // case["page_rows"])
    have = -(-before // case["page_rows"])
    spare = int(np.maximum(need - have, 0).sum()) + 7
    table, free, n_pages = _random_pages(before, case["page_rows"], case["cols"], spare, seed)
    init = _page_state(table, before, free, n_pages)
    return {"case": case, "init": init, "work": init.clone(), "n_pages": n_pages,
            "target": torch.from_numpy(after.astype(np.int32)).cuda(),
            "slots": torch.zeros((case["requests"], case["max_new"]), dtype=torch.int64, device="cuda")}


def _prepare_rows(case, seed, g):
    b, cap, pr = case["requests"], case["cap"], case["page_rows"]
    n_new = _spread_in_turn(case["rows_lo"], case["rows_hi"], b, seed)
    start = _spread_in_turn(case["start_lo"], case["start_hi"], b, seed + 2)
    cols = int(-(-(start + n_new).max() // pr)) + 1
    table, free, n_pages = _random_pages(start + n_new, pr, cols, 3, seed)
    at = start[:, None] + np.arange(cap)[None, :]
    slots = table[np.arange(b)[:, None], np.minimum(at // pr, cols - 1)].astype(np.int64) * pr + at % pr
    slots[np.arange(cap)[None, :] >= n_new[:, None]] = -1
    l, h, d, dt = case["layers"], case["kv_heads"], case["head_dim"], _DTYPES[case["dtype"]]
    stride = h * d + case["pad"]
    # a few channels of the keys are large in every row, as in trained models
    loud = torch.where(torch.rand(h * d, generator=g, device="cuda") < 0.05, 6.0, 1.0)
    k = torch.zeros((l, b, cap, stride), dtype=dt, device="cuda")
    v = torch.zeros_like(k)
    k[..., :h * d] = _normal((l, b, cap, h * d), g) * loud
    v[..., :h * d] = _normal((l, b, cap, h * d), g) * 0.3
    pool = torch.zeros((l, n_pages, h, pr // 16, 18 * d), dtype=torch.uint8, device="cuda")
    back = torch.zeros((2, l, b, cap, h, d), dtype=dt, device="cuda")
    return {"case": case, "k": k[..., :h * d].unflatten(-1, (h, d)), "v": v[..., :h * d].unflatten(-1, (h, d)), "pool": pool, "back": back,
            "slots": torch.from_numpy(slots).cuda(), "n_pages": n_pages}


def _prepare_attn(case, seed, g):
    b, pr, l, h, d = case["requests"], case["page_rows"], case["layers"], case["kv_heads"], case["head_dim"]
    rows = _spread_in_turn(case["rows_lo"], case["rows_hi"], b, seed)
    cols = int(-(-rows.max() // pr)) + 2
    table, free, n_pages = _random_pages(rows, pr, cols, 3, seed)
    pool = torch.empty((l, n_pages, h, pr // 16, 18 * d), dtype=torch.uint8, device="cuda")
    loud = torch.where(torch.rand((h, 1, d), generator=g, device="cuda") < 0.05, 3.0, 1.0)
    for layer in range(l):
        for p0 in range(0, n_pages, max(1, (1 << 27) // (h * pr * d))):
            part = pool[layer, p0:p0 + max(1, (1 << 27) // (h * pr * d))]
            shape = (part.shape[0], h, pr, d)
            part.copy_(_blocks(_normal(shape, g) * loud, _normal(shape, g)))
    q = _normal((l, b, case["q_len"], case["q_heads"], d), g, _DTYPES[case["dtype"]])
    case = dict(case, cols=cols)
    return {"case": case, "pool": pool, "q": q, "state": _page_state(table, rows, free, n_pages), "n_pages": n_pages}


# -------------------------------------------------------------------------------------------------- plain forms

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"pages": _own_pages, "rows": _own_rows, "attn": _own_attn}[kind](state)
    return {"pages": _plain_pages, "rows": _plain_rows, "attn": _plain_attn}[kind](state)


def _plain_pages(s):
    """Releases first, last request and column first, so that growing and shrinking back leaves the stack as it was; then
    the growing requests take pages in order, each only if all it needs is left."""
    case = s["case"]
    s["work"].copy_(s["init"])
    table, rows, free, count, status = _views(case, s["work"], s["n_pages"])
    b, cols, pr = case["requests"], case["cols"], case["page_rows"]
    after = torch.clamp(s["target"].long(), min=0)
    before = rows.long()
    have, need = (before + pr - 1) // pr, (after + pr - 1) // pr
    col = torch.arange(cols, device="cuda")[None, :]
    freed = ((col >= need[:, None]) & (col < have[:, None])).flatten().flip(0)
    height = count.long() + torch.cumsum(freed, 0)[-1:]
    at = torch.where(freed, count.long() + torch.cumsum(freed, 0) - 1, s["n_pages"])
    stack = torch.cat([free.long(), torch.zeros(1, dtype=torch.int64, device="cuda")])
    stack = stack.scatter(0, at, table.flatten().flip(0).long())
    fits = (after <= cols * pr) & (after - before <= case["max_new"])
    wants = torch.where(fits, torch.clamp(need - have, min=0), 0)
    total = torch.cumsum(wants, 0)
    served = fits & ((wants == 0) | (total <= height))
    taken = served[:, None] & (col >= have[:, None]) & (col < need[:, None])
    from_top = (total - wants)[:, None] + col - have[:, None]
    page = stack[torch.clamp(height - 1 - from_top, min=0, max=s["n_pages"] - 1)]
    gone = (col >= need[:, None]) & (col < have[:, None])
    new_table = torch.where(taken, page, torch.where(gone, -1, table.long()))
    new_rows = torch.where(served, after, before)
    left = height - torch.where(served, wants, 0).sum()
    i = torch.arange(case["max_new"], device="cuda")[None, :]
    row = before[:, None] + i
    page = torch.gather(new_table, 1, torch.clamp(row // pr, max=cols - 1))
    s["slots"].copy_(torch.where(row < new_rows[:, None], page * pr + row % pr, -1))
    table.copy_(new_table)
    rows.copy_(new_rows)
    free.copy_(stack[:-1])
    count.copy_(left)
    return _pages_answer(s, table, rows, free, count)


def _pages_answer(s, table, rows, free, count):
    """The stack is what lies below its height: what is above is left as it comes."""
    return {"table": table, "rows": rows, "count": count, "slots": s["slots"],
            "free": torch.where(torch.arange(s["n_pages"], device="cuda") < count, free, -1)}


def _quantise(x: torch.Tensor):
    """(codes uint8 [..., d], scales bf16 [..., d / 32]) of x [..., d]."""
    x = x.float().unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1)
    scale = (amax / 6.0).to(torch.bfloat16).float()
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    y = x.abs() / torch.where(scale > 0, scale, 1.0)[..., None]
    code = ((y > 0.25).byte() + (y >= 0.75).byte() + (y > 1.25).byte() + (y >= 1.75).byte() + (y > 2.5).byte() + (y >= 3.5).byte() +
            (y > 5.0).byte())
    code = torch.where((scale > 0)[..., None], code | (torch.signbit(x).byte() << 3), 0).byte()
    bad = ~torch.isfinite(amax)
    code = torch.where(bad[..., None], 0, code).byte()
    return code.flatten(-2), torch.where(bad, float("nan"), scale).to(torch.bfloat16)


def _split(blocks: torch.Tensor):
    """Views of a pool's blocks [..., 18 d]: key codes [..., row, t, group, 4] (byte i holds numbers 32 group + 8 t + 2 i and
    the next one, the first in its low half), value codes [..., half, u, t, odd, group, 2] (row 8 half + 2 t + odd, byte i holds
    numbers 32 group + 4 u + 2 i and the next one), scales [..., row, group] of the keys and of the values."""
    d = blocks.shape[-1] // 18
    lead = blocks.shape[:-1]
    return (blocks[..., :8 * d].unflatten(-1, (16, 4, d // 32, 4)), blocks[..., 8 * d:16 * d].unflatten(-1, (2, 8, 4, 2, d // 32, 2)),
            blocks[..., 16 * d:17 * d].view(torch.bfloat16).view(*lead, 16, d // 32),
            blocks[..., 17 * d:].view(torch.bfloat16).view(*lead, 16, d // 32))


def _blocks(k: torch.Tensor, v: torch.Tensor) -> torch.Tensor:
    """Pool bytes [..., rows / 16, 18 d] of keys and values [..., rows, d]."""
    d = k.shape[-1]
    out = torch.empty(k.shape[:-2] + (k.shape[-2] // 16, 18 * d), dtype=torch.uint8, device=k.device)
    kc, vc, ks, vs = _split(out)
    code, scale = _quantise(k)
    code = code.unflatten(-2, (-1, 16)).unflatten(-1, (d // 32, 4, 4, 2)).movedim(-4, -3)        # row, t, group, byte, half
    kc.copy_(code[..., 0] | (code[..., 1] << 4))
    ks.copy_(scale.unflatten(-2, (-1, 16)))
    code, scale = _quantise(v)
    code = code.unflatten(-2, (-1, 2, 4, 2)).unflatten(-1, (d // 32, 8, 2, 2))                   # half, t, odd, group, u, byte, half
    code = code.movedim(-3, -6)
    vc.copy_(code[..., 0] | (code[..., 1] << 4))
    vs.copy_(scale.unflatten(-2, (-1, 16)))
    return out


def _numbers(blocks: torch.Tensor):
    """fp32 keys and values [..., 16, d] of blocks [..., 18 d]."""
    d = blocks.shape[-1] // 18
    kc, vc, ks, vs = _split(blocks)
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=blocks.device)
    k = level[torch.stack([kc & 15, kc >> 4], -1).int()]                                           # row, t, group, byte, half
    k = k.movedim(-4, -3).flatten(-3)                                                              # row, group, 32
    v = level[torch.stack([vc & 15, vc >> 4], -1).int()]                                           # half, u, t, odd, group, byte, half
    v = v.movedim(-6, -3).flatten(-3)                                                              # half, t, odd, group, 32
    v = v.flatten(-5, -3)
    return (k * ks.float()[..., None]).flatten(-2), (v * vs.float()[..., None]).flatten(-2)


def _plain_rows(s):
    """Rows to their slots, and back.  The slots' blocks are taken as rows of numbers' codes: a row's bytes lie at fixed places."""
    case, pool = s["case"], s["pool"]
    l, h, d, pr = case["layers"], case["kv_heads"], case["head_dim"], case["page_rows"]
    slots = s["slots"].flatten()
    kept = torch.nonzero(slots >= 0).flatten()
    slot = slots[kept]
    page, block, row = slot // pr, slot % pr // 16, slot % 16
    k = s["k"].flatten(1, 2)[:, kept]
    v = s["v"].flatten(1, 2)[:, kept]
    kc, vc, ks, vs = _split(pool)                                   # [l, page, h, block, row, ...]
    head = torch.arange(h, device="cuda")
    code, scale = _quantise(k)                                      # [l, n, h, d]
    code = code.unflatten(-1, (d // 32, 4, 4, 2)).movedim(-4, -3)
    at = (page[:, None], head[None, :], block[:, None], row[:, None])
    kc[(slice(None),) + at] = code[..., 0] | (code[..., 1] << 4)
    ks[(slice(None),) + at] = scale
    code, scale = _quantise(v)
    code = code.unflatten(-1, (d // 32, 8, 2, 2)).movedim(-4, -3)   # u, group, byte, half
    vt = vc.movedim(-5, -3)                                         # [l, page, h, block, half, t, odd, u, group, 2]
    spot = at[:3] + (row[:, None] // 8, row[:, None] % 8 // 2, row[:, None] % 2)
    vt[(slice(None),) + spot] = code[..., 0] | (code[..., 1] << 4)
    vs[(slice(None),) + at] = scale
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device="cuda")
    back = s["back"]
    got = kc[(slice(None),) + at]
    x = level[torch.stack([got & 15, got >> 4], -1).int()].movedim(-4, -3).flatten(-3)
    back[0].flatten(1, 2)[:, kept] = (x * ks[(slice(None),) + at].float()[..., None]).flatten(-2).to(back.dtype)
    got = vt[(slice(None),) + spot]
    x = level[torch.stack([got & 15, got >> 4], -1).int()].movedim(-4, -3).flatten(-3)
    back[1].flatten(1, 2)[:, kept] = (x * vs[(slice(None),) + at].float()[..., None]).flatten(-2).to(back.dtype)
    return {"k": back[0], "v": back[1]}


def _plain_attn(s):
    case = s["case"]
    l, b, h, d, pr, n = case["layers"], case["requests"], case["kv_heads"], case["head_dim"], case["page_rows"], case["q_len"]
    grp = case["q_heads"] // h
    table, rows = _views(case, s["state"], s["n_pages"])[:2]
    blocks = s["pool"][:, torch.clamp(table, min=0)]                 # [l, b, cols, h, blocks, 18 d]
    k, v = _numbers(blocks.movedim(3, 2))                            # [l, b, h, cols, blocks, 16, d]
    k, v = k.flatten(3, 5), v.flatten(3, 5)
    q = s["q"].float().unflatten(3, (h, grp)).permute(0, 1, 3, 4, 2, 5).flatten(3, 4)   # [l, b, h, grp * n, d]
    x = q @ k.transpose(-1, -2) / math.sqrt(d)
    sees = rows.long()[:, None] - n + 1 + torch.arange(n, device="cuda")[None, :]       # [b, n]
    mask = torch.arange(k.shape[3], device="cuda") < sees[..., None]                    # [b, n, keys]
    mask = mask[None, :, None, None].expand(l, b, h, grp, n, -1).flatten(3, 4)
    x = torch.where(mask, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.where(mask, torch.exp(x - torch.where(m == -math.inf, 0.0, m)), 0.0)
    total = p.sum(-1, keepdim=True)
    # rows behind the last are left out of the sums, whatever they hold
    v = torch.where((torch.arange(k.shape[3], device="cuda") < rows[:, None])[None, :, None, :, None], v, 0.0)
    out = torch.where(total > 0, (p @ v) / torch.where(total > 0, total, 1.0), 0.0)
    lse = (m + torch.log(total))[..., 0]
    out = out.unflatten(3, (grp, n)).permute(0, 1, 4, 2, 3, 5).flatten(3, 4).to(s["q"].dtype)
    return {"out": out, "lse": lse.unflatten(3, (grp, n)).flatten(2, 3)}                 # [l, b, q_heads, n]


# ---------------------------------------------------------------------------------------- through the library

def _handle(s, flat):
    """What a program keeps: the descriptors of its model and of its pages."""
    import paper_2502_11101_b200 as cf
    case = s["case"]
    table, rows, free, count, status = _views(case, flat, s["n_pages"])
    made = {"cf": cf, "pages": cf.make_pages(table, rows, free, count, status, case["page_rows"]), "views": (table, rows, free, count),
            "place": torch.arange(s["n_pages"], device="cuda")}
    if "head_dim" in case:
        made["geom"] = cf.make_geom(case.get("q_heads", case["kv_heads"]), case["kv_heads"], case["head_dim"], _DTYPES[case["dtype"]], 32768, 1.0e6)
    return made


def _own_pages(s):
    if "handle" not in s:
        s["handle"] = _handle(s, s["work"])
    hd = s["handle"]
    s["work"].copy_(s["init"])
    hd["cf"].cf_pages_resize(hd["pages"], s["target"], 0, s["slots"])
    table, rows, free, count = hd["views"]
    return {"table": table, "rows": rows, "count": count, "slots": s["slots"], "free": torch.where(hd["place"] < count, free, -1)}


def _own_rows(s):
    if "handle" not in s:
        cols = 1
        case = dict(s["case"], cols=cols)
        flat = _page_state(np.full((case["requests"], cols), -1, np.int32), np.zeros(case["requests"]), np.zeros(0, np.int32), s["n_pages"])
        s["handle"] = _handle(dict(s, case=case), flat)
        s["flat"] = flat
    hd = s["handle"]
    hd["cf"].cf_kv4_write(hd["geom"], hd["pages"], s["pool"], s["slots"], s["k"], s["v"])
    hd["cf"].cf_kv4_read(hd["geom"], hd["pages"], s["pool"], s["slots"], s["back"][0], s["back"][1])
    return {"k": s["back"][0], "v": s["back"][1]}


def _own_attn(s):
    case, q = s["case"], s["q"]
    if "handle" not in s:
        hd = s["handle"] = _handle(s, s["state"])
        need = hd["cf"].cf_kv4_attn_workspace_bytes(hd["geom"], hd["pages"], case["q_len"], case["layers"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        s["out"] = torch.empty_like(q)
        s["lse"] = torch.empty((case["layers"], case["requests"], case["q_heads"], case["q_len"]), device="cuda")
    hd = s["handle"]
    hd["cf"].cf_kv4_attn(hd["geom"], hd["pages"], s["pool"], q, s["out"], s["workspace"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------------- work

def work(case: Dict) -> Dict:
    """Attention: codes and scales of the rows in use once, queries and results once; two products.  Rows: the numbers in and
    out, codes and scales written and read.  Pages: lengths in and out, the entries that change, the slot map."""
    if case["kind"] == "pages":
        before, after = _targets(case)
        pr = case["page_rows"]
        moved = int(np.abs(-(-np.maximum(after, 0) // pr) - -(-before // pr)).sum())
        n = case["requests"]
        return {"bytes": 12 * n + 8 * moved + 8 * n * case["max_new"], "flops": 0}
    d, h, l = case["head_dim"], case["kv_heads"], case["layers"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rows":
        rows = int(_spread(case["rows_lo"], case["rows_hi"], case["requests"]).sum()) * l * h
        return {"bytes": rows * (2 * 2 * d * size + 2 * 2 * (d // 2 + d // 16)) + 2 * 8 * case["requests"] * case["cap"], "flops": 6 * rows * 2 * d}
    lengths = _spread(case["rows_lo"], case["rows_hi"], case["requests"])
    n, grp = case["q_len"], case["q_heads"] // h
    seen = int(sum(np.maximum(lengths - j, 0).sum() for j in range(n)))
    return {"bytes": int(lengths.sum()) * l * h * 2 * (d // 2 + d // 16) + l * case["requests"] * n * case["q_heads"] * (2 * d * size + 4),
            "flops": 4 * d * seen * h * grp * l}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_value(x: torch.Tensor) -> torch.Tensor:
    """What the format keeps of x [..., d], by searching the nearest number that it has."""
    x = x.double()
    grouped = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    ideal = grouped.abs().max(dim=-1).values / 6.0
    fraction, power = torch.frexp(torch.where(ideal > 0, ideal, torch.ones_like(ideal)))
    scale = torch.ldexp(torch.round(fraction * 256.0), power - 8)       # eight bits, ties to even
    scale = torch.where(ideal > 0, scale, torch.zeros_like(ideal))
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    kept = torch.zeros_like(grouped)
    near = torch.full_like(grouped, math.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):                               # even codes first: they keep a tie
        off = (grouped.abs() - _LEVELS[code] * scale[..., None]).abs()
        better = off < near
        near = torch.where(better, off, near)
        kept = torch.where(better, _LEVELS[code] * scale[..., None], kept)
    return (torch.sign(grouped) * kept).reshape(x.shape)


def _exact_rows(pool_page: torch.Tensor, d: int):
    """Keys and values [h, rows, d] in 64 bits of one page [h, blocks, 18 d], every code looked up where the format puts it."""
    h, nb = pool_page.shape[:2]
    dim = torch.arange(d, device="cuda")
    row = torch.arange(16, device="cuda")[:, None]
    group, rest = dim // 32, dim % 32
    k_at = row * (d // 2) + (rest // 8) * (d // 8) + group * 4 + (rest % 8) // 2
    v_at = 8 * d + (row // 8) * (4 * d) + (rest // 4) * (d // 2) + ((row % 8) // 2) * (d // 8) + (row % 2) * (d // 16) + group * 2 + (rest % 4) // 2
    value = torch.tensor([s * x for s in (1.0, -1.0) for x in _LEVELS], dtype=torch.float64, device="cuda")
    found = []
    for at, scales_at in ((k_at, 16 * d), (v_at, 17 * d)):
        byte = pool_page[:, :, at.reshape(-1)].reshape(h, nb, 16, d).long()
        code = (byte >> (4 * (dim % 2))) & 15
        scale = pool_page[:, :, scales_at:scales_at + d].contiguous().view(torch.bfloat16).double().reshape(h, nb, 16, d // 32)
        found.append((value[code] * scale[..., group]).reshape(h, nb * 16, d))
    return found


def exact(case: Dict, seed: int):
    s = prepare(case, seed)
    if case["kind"] == "pages":
        return None
    if case["kind"] == "rows":
        keep = (s["slots"] >= 0)[None, :, :, None, None]
        return {n: torch.where(keep, torch.stack([_exact_value(x) for x in s[n]]), 0.0) for n in ("k", "v")}
    full, d, n = s["case"], case["head_dim"], case["q_len"]
    if case["layers"] * case["requests"] * n > 4000:
        return None
    table, rows = (t.cpu() for t in _views(full, s["state"], s["n_pages"])[:2])
    grp, pr = case["q_heads"] // case["kv_heads"], case["page_rows"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full((case["layers"], case["requests"], case["q_heads"], n), -math.inf, dtype=torch.float64, device="cuda")
    for layer in range(case["layers"]):
        for b in range(case["requests"]):
            used = int(rows[b])
            if used == 0:
                continue
            pages = table[b, :-(-used // pr)].long().cuda()
            got = s["pool"][layer, pages].transpose(0, 1).reshape(case["kv_heads"], -1, 18 * d)
            k, v = (x[:, :used] for x in _exact_rows(got, d))
            for j in range(n):
                sees = used - n + 1 + j
                if sees <= 0:
                    continue
                q = s["q"][layer, b, j].double().reshape(case["kv_heads"], grp, d)
                x = torch.einsum("hgd,hkd->hgk", q, k[:, :sees]) * d ** -0.5
                lse[layer, b, :, j] = torch.logsumexp(x, -1).reshape(-1)
                out[layer, b, j] = torch.einsum("hgk,hkd->hgd", torch.softmax(x, -1), v[:, :sees]).reshape(-1, d)
    return {"out": out, "lse": lse}
