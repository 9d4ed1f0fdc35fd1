"""What the speed of the engine-step operators is measured on: slot maps, rotary rows with their append, whole-prompt
attention.

A case is one call of a public entry point of ``paper_2609_08368_amd.rl_attn``. ``op`` names the call:

* "map": block tables, slot map and positions of a step from its request lengths (``map_slots``);
* "rope": rotary positions with one or several axes on query and key rows (``rope``);
* "rope_append": the same in one pass with the append of the step's rows to their pages (``rope_append_kv`` or, with
  ``fp8``, ``rope_append_kv_fp8``);
* "prefill": causal attention over whole packed prompts (``prefill``).

Lengths are drawn from ``shape_seed``, so a case always has the same shape; values, positions and page order come from
the seed of the preparation. ``own`` selects the framework's calls; without it ``run`` computes the same in plain torch
operations.
"""

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
D = 128                          # head dimension
MOST_SCORES = 64 * 16384 ** 2    # padded scores of the largest prefill, which the plain form holds in memory
MOST_ROPE = 36098 * 88           # (row, head) pairs of the largest rope call
MOST_ROWS = 65536                # rows of the largest slot map
MOST_TABLE = 1 << 22             # entries of the largest block table

# every field a case may leave out
DEFAULTS = {
    "lse": False,                # prefill: the log-sum-exp is asked for too
    "pad": 0,                    # rows behind the last request's (a batch padded to a captured size)
    "fp8": False,                # rope_append: E4M3 pages with one scale per KV head
    "k_out": False,              # rope_append: the rotated keys are wanted as rows too
    "axes": "",                  # rope: "" one axis, "blocks" or "cycle": three, by blocks of frequencies or in turn
    "rotated": D,                # rope: dimensions that are rotated
    "interleaved": False,        # rope: pairs of neighbours instead of halves
    "inverse": False,            # rope: rotated back (also the gradient)
    "far": 0,                    # rope: positions start here
    "page": 64,
    "delta": False,              # map: positions differ from the cached length (after images)
}


def listed():
    return [
        # a decode step of the 128 agentic sessions: one new token each, a page filled now and then
        {"name": "map_decode", "op": "map", "batch": 128, "cached_lo": 1024, "cached_hi": 65536, "new_lo": 1,
         "new_hi": 1, "shape_seed": 1, "delta": True},
        # the multi-turn batch: 32 sessions append turns of 64 to 2048 tokens
        {"name": "map_turns", "op": "map", "batch": 32, "cached_lo": 8192, "cached_hi": 65536, "new_lo": 64,
         "new_hi": 2048, "shape_seed": 1005},
        # many short requests in small pages, some with nothing new, padded to a captured size
        {"name": "map_many", "op": "map", "batch": 3001, "cached_lo": 0, "cached_hi": 900, "new_lo": 0, "new_hi": 33,
         "page": 16, "shape_seed": 2, "pad": 777},
        # the same decode step's rows on a 96/8-head model, far positions, text beside images
        {"name": "rope_append_decode", "op": "rope_append", "rows": 128, "hq": 96, "hkv": 8, "axes": "blocks",
         "far": 60000, "shape_seed": 3},
        # the multi-turn batch's 36K rows, whose keys are wanted as rows too
        {"name": "rope_append_turns", "op": "rope_append", "rows": 36098, "hq": 64, "hkv": 8, "axes": "cycle",
         "k_out": True, "shape_seed": 4},
        # an odd number of rows into an FP8 cache, padded to a captured size
        {"name": "rope_append_fp8", "op": "rope_append", "rows": 9999, "hq": 64, "hkv": 8, "fp8": True, "pad": 241,
         "shape_seed": 5},
        # a small model with half of each head rotated, pairs of neighbours, gradients on their way back
        {"name": "rope_back", "op": "rope", "rows": 1777, "hq": 8, "hkv": 2, "rotated": 64, "interleaved": True,
         "inverse": True, "shape_seed": 6},
        # one short prompt on a small model: latency
        {"name": "prefill_one", "op": "prefill", "batch": 1, "hq": 8, "hkv": 2, "len_lo": 37, "len_hi": 37,
         "shape_seed": 7},
        # a handful of odd prompts with their log-sum-exp, rows behind them
        {"name": "prefill_odd", "op": "prefill", "batch": 24, "hq": 96, "hkv": 8, "len_lo": 0, "len_hi": 701,
         "lse": True, "pad": 100, "shape_seed": 8},
        # the prompts of 16 trajectory groups, up to 4096 tokens
        {"name": "prefill_groups", "op": "prefill", "batch": 16, "hq": 64, "hkv": 8, "len_lo": 2000, "len_hi": 4096,
         "shape_seed": 9},
        # a prompt of 4096 tokens on a model with few heads: little to spread over the device
        {"name": "prefill_few_heads", "op": "prefill", "batch": 1, "hq": 8, "hkv": 2, "len_lo": 4095, "len_hi": 4095,
         "shape_seed": 10},
        # one long prompt
        {"name": "prefill_long", "op": "prefill", "batch": 1, "hq": 64, "hkv": 8, "len_lo": 16384, "len_hi": 16384,
         "shape_seed": 11},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any mix of heads, formats and options, sizes over the logarithm of their range."""
    op = rng.choice(["map", "rope", "rope_append", "rope_append", "prefill", "prefill", "prefill"])
    c = {"op": op, "shape_seed": rng.randrange(1 << 20)}
    hq, hkv = rng.choice([(8, 2), (32, 8), (64, 8), (64, 8), (96, 8), (16, 16), (8, 1), (12, 1)])
    pad = rng.choice([0, 0, rng.randrange(1, 300)])
    if op == "map":
        batch = _log_int(rng, 1, 4096)
        hi = max(1, min(_log_int(rng, 1, 2048), MOST_ROWS // batch))
        page = rng.choice([8, 16, 32, 64, 64, 128])
        cached = min(_log_int(rng, 64, 65536), max(1, MOST_TABLE // batch * page - hi - page))
        c.update(batch=batch, new_lo=rng.choice([0, 1, hi]), new_hi=hi, cached_lo=rng.choice([0, cached // 2]),
                 cached_hi=cached, page=page, pad=pad, delta=rng.random() < 0.5)
        c["new_lo"] = min(c["new_lo"], hi)
    elif op == "prefill":
        batch = _log_int(rng, 1, 64)
        hi = min(_log_int(rng, 1, 16384), int(math.sqrt(MOST_SCORES / hq / batch)))
        c.update(batch=batch, hq=hq, hkv=hkv, len_lo=rng.choice([0, 1, hi // 2, hi]), len_hi=hi, pad=pad,
                 lse=rng.random() < 0.4)
        c["len_lo"] = min(c["len_lo"], hi)
    else:
        c.update(rows=_log_int(rng, 1, min(65536, MOST_ROPE // (hq + 3 * hkv))), hq=hq, hkv=hkv,
                 axes=rng.choice(["", "blocks", "cycle"]), rotated=rng.choice([D, D, 96, 64, 32]),
                 interleaved=rng.random() < 0.3, far=rng.choice([0, _log_int(rng, 100, 1 << 20)]))
        if op == "rope":
            c["inverse"] = rng.random() < 0.5
        else:
            c.update(page=rng.choice([8, 16, 32, 64, 64, 128]), fp8=rng.random() < 0.4, k_out=rng.random() < 0.4,
                     pad=pad)
    return c


def _full(case):
    return {**DEFAULTS, **case}


def _lens(c, lo, hi, salt=0):
    """Lengths of a case's requests; a range from 0 on has an empty request for certain."""
    rng = np.random.default_rng(1000 * c["shape_seed"] + salt)
    n = rng.integers(lo, hi + 1, size=c["batch"])
    n[int(rng.integers(c["batch"]))] = hi
    if lo == 0 and c["batch"] > 1:
        n[(int(np.argmax(n)) + 1) % c["batch"]] = 0
    return n.astype(np.int64)


def _dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEVICE, dtype=dtype)


def _normal(seed, shape):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEVICE).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ preparation

def prepare(case, seed):
    c = _full(case)
    s = {"case": c}
    {"map": _prepare_map, "rope": _prepare_rope, "rope_append": _prepare_rope, "prefill": _prepare_prefill}[c["op"]](
        c, seed, s)
    return s


def _prepare_map(c, seed, s):
    rng = np.random.default_rng(seed)
    page, batch = c["page"], c["batch"]
    cached, new = _lens(c, c["cached_lo"], c["cached_hi"], 1), _lens(c, c["new_lo"], c["new_hi"], 2)
    before, after = -(-cached // page), -(-(cached + new) // page)
    width = int(after.max()) + 3
    pool = int(after.sum()) + 50
    ids = rng.permutation(pool)
    table = np.full((batch, width), -1, np.int64)
    held = np.arange(width)[None, :] < before[:, None]
    table[held] = ids[:int(before.sum())]
    used = int(rng.integers(0, 40))                      # entries of the free list that earlier steps took
    free = np.concatenate([rng.integers(0, pool, used), ids[int(before.sum()):]])
    rows = int(new.sum()) + c["pad"]
    s.update(kv_lens=_dev(cached, torch.int32), new_lens=_dev(new, torch.int32), free_pages=_dev(free, torch.int32),
             free_used=_dev(np.array([used]), torch.int32), block_table=_dev(table, torch.int32), pages=pool,
             rows=rows, total=int(new.sum()), width=width,
             delta=_dev(rng.integers(-900, 5, batch), torch.int32) if c["delta"] else None,
             kv_out=torch.zeros(batch, dtype=torch.int32, device=DEVICE),
             used_out=torch.zeros(1, dtype=torch.int32, device=DEVICE),
             indptr=torch.zeros(batch + 1, dtype=torch.int32, device=DEVICE),
             slot_map=torch.zeros(rows, dtype=torch.int64, device=DEVICE),
             positions=torch.zeros(rows, dtype=torch.int32, device=DEVICE))


def _positions(c, seed, rows):
    """Positions of a stream of text and images: a text token moves all three axes on, an image holds time and walks
    its rows and columns."""
    rng = np.random.default_rng(seed)
    if not c["axes"]:
        return c["far"] + np.arange(rows) + rng.integers(0, 100)
    parts, at, have = [], c["far"] + int(rng.integers(0, 100)), 0
    while have < rows:
        n = int(rng.integers(1, 400))
        parts.append(np.tile(at + np.arange(n), (3, 1)))
        at, have = at + n, have + n
        h, w = int(rng.integers(2, 40)), int(rng.integers(2, 40))
        grid = np.indices((h, w)).reshape(2, -1)
        parts.append(np.stack([np.zeros(h * w, np.int64), grid[0], grid[1]]) + at)
        at, have = at + max(h, w), have + h * w
    return np.concatenate(parts, axis=1)[:, :rows]


def _prepare_rope(c, seed, s):
    rng = np.random.default_rng(seed + 1)
    rows, hq, hkv, page = c["rows"] + c["pad"], c["hq"], c["hkv"], c["page"]
    f = c["rotated"] // 2
    qkv = _normal(seed, (rows, hq + 2 * hkv, D))         # as a fused projection leaves them
    axis = {"": None, "blocks": np.repeat([0, 1, 2], [f - 2 * (3 * f // 8), 3 * f // 8, 3 * f // 8]),
            "cycle": np.arange(f) % 3}[c["axes"]]
    pos = _positions(c, seed + 2, rows)
    s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], real=c["rows"],
             positions=_dev(pos.reshape(-1, rows), torch.int32),
             inv_freq=_dev(1e6 ** (-np.arange(f) / f), torch.float32),
             axes=None if axis is None else _dev(axis, torch.int32),
             q_out=torch.zeros((rows, hq, D), dtype=torch.bfloat16, device=DEVICE),
             k_rows=torch.zeros((rows, hkv, D), dtype=torch.bfloat16, device=DEVICE))
    if c["op"] == "rope":
        return
    pool = -(-c["rows"] // page) + 7
    order = rng.permutation(pool)
    at = np.arange(c["rows"]) + int(rng.integers(0, page))
    slots = np.concatenate([order[at // page] * page + at % page, np.full(c["pad"], -1)])
    kind = torch.float8_e4m3fn if c["fp8"] else torch.bfloat16
    s.update(slot_map=_dev(slots, torch.int64),
             k_pages=torch.zeros((pool, page, hkv, D), dtype=kind, device=DEVICE),
             v_pages=torch.zeros((pool, page, hkv, D), dtype=kind, device=DEVICE),
             k_scale=_dev(rng.uniform(0.008, 0.02, hkv), torch.float32),
             v_scale=_dev(rng.uniform(0.008, 0.02, hkv), torch.float32))


def _prepare_prefill(c, seed, s):
    lens = _lens(c, c["len_lo"], c["len_hi"])
    indptr = np.concatenate([[0], np.cumsum(lens)])
    rows, hq, hkv = int(indptr[-1]) + c["pad"], c["hq"], c["hkv"]
    qkv = _normal(seed, (rows, hq + 2 * hkv, D))
    g = np.random.default_rng(seed).uniform(0.5, 2.0, hkv)     # heads of different sharpness
    qkv[:, hq:hq + hkv] *= _dev(g, torch.bfloat16)[None, :, None]
    s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], indptr=_dev(indptr, torch.int32),
             scale=1.0 / math.sqrt(D), longest=int(lens.max()), real=int(indptr[-1]),
             out=torch.zeros((rows, hq, D), dtype=torch.bfloat16, device=DEVICE),
             lse=torch.zeros((rows, hq), dtype=torch.float32, device=DEVICE) if c["lse"] else None)


# ------------------------------------------------------------------------------------------------------- runs

def run(state):
    return {"map": _run_map, "rope": _run_rope, "rope_append": _run_rope_append, "prefill": _run_prefill}[
        state["case"]["op"]](state)


def _map_answer(s):
    return {"block_table": s["block_table"], "kv_lens": s["kv_out"], "free_used": s["used_out"], "indptr": s["indptr"],
            "slot_map": s["slot_map"], "positions": s["positions"]}


def _run_map(s):
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        ra.map_slots(s["kv_lens"], s["new_lens"], s["free_pages"], s["free_used"], s["block_table"],
                     s["case"]["page"], s["pages"], pos_delta=s["delta"], kv_lens_out=s["kv_out"],
                     free_used_out=s["used_out"], qo_indptr=s["indptr"], slot_map=s["slot_map"],
                     positions=s["positions"])
        return _map_answer(s)
    page, total, cached, new = s["case"]["page"], s["total"], s["kv_lens"].long(), s["new_lens"].long()
    after = cached + new
    before_pages, after_pages = (cached + page - 1) // page, (after + page - 1) // page
    need = after_pages - before_pages
    s["kv_out"].copy_(after)
    s["used_out"].copy_(s["free_used"] + need.sum())
    s["indptr"][1:] = torch.cumsum(new, 0)
    first = s["free_used"] + torch.cumsum(need, 0) - need
    b = torch.repeat_interleave(torch.arange(len(new), device=DEVICE), new, output_size=total)
    t = cached[b] + torch.arange(total, device=DEVICE) - (torch.cumsum(new, 0) - new)[b]
    j = t // page
    fresh = j - before_pages[b]
    taken = s["free_pages"][(first[b] + fresh).clamp(0, s["free_pages"].shape[0] - 1)]
    ids = torch.where(fresh >= 0, taken, s["block_table"][b, j])
    s["block_table"][b, j] = ids
    s["slot_map"].fill_(-1)
    s["slot_map"][:total] = ids.long() * page + t % page
    s["positions"].zero_()
    s["positions"][:total] = t if s["delta"] is None else t + s["delta"][b]
    return _map_answer(s)


def _angles(s, dtype):
    """cos and sin [rows, 1, F] of position times frequency: the angle in 64 bits, where far positions need them."""
    pos = s["positions"].double()
    which = s["axes"].long() if s["axes"] is not None else torch.zeros(s["inv_freq"].shape[0], dtype=torch.long,
                                                                       device=DEVICE)
    a = pos[which].T * s["inv_freq"].double()
    a = -a if s["case"]["inverse"] else a
    return a.cos().to(dtype)[:, None], a.sin().to(dtype)[:, None]


def _rotate(x, cos, sin, f, interleaved):
    x = x.to(cos.dtype)
    if interleaved:
        a, b = x[..., 0:2 * f:2], x[..., 1:2 * f:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :f], x[..., f:2 * f]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, x[..., 2 * f:]), dim=-1)


def _run_rope(s):
    c = s["case"]
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        ra.rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["axes"], interleaved=c["interleaved"],
                inverse=c["inverse"], q_out=s["q_out"], k_out=s["k_rows"])
    else:
        cos, sin = _angles(s, torch.float32)
        f = s["inv_freq"].shape[0]
        s["q_out"].copy_(_rotate(s["q"], cos, sin, f, c["interleaved"]))
        s["k_rows"].copy_(_rotate(s["k"], cos, sin, f, c["interleaved"]))
    return {"q": s["q_out"], "k": s["k_rows"]}


def _rope_answer(s):
    out = {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return {**out, "k": s["k_rows"]} if s["case"]["k_out"] else out


def _run_rope_append(s):
    c = s["case"]
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        k_out = s["k_rows"] if c["k_out"] else None
        if c["fp8"]:
            ra.rope_append_kv_fp8(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["slot_map"], s["k_pages"],
                                  s["v_pages"], s["k_scale"], s["v_scale"], s["axes"], interleaved=c["interleaved"],
                                  q_out=s["q_out"], k_out=k_out)
        else:
            ra.rope_append_kv(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["slot_map"], s["k_pages"],
                              s["v_pages"], s["axes"], interleaved=c["interleaved"], q_out=s["q_out"], k_out=k_out)
        return _rope_answer(s)
    n, f = s["real"], s["inv_freq"].shape[0]
    cos, sin = _angles(s, torch.float32)
    k = _rotate(s["k"], cos, sin, f, c["interleaved"])[:n]
    s["q_out"][:n] = _rotate(s["q"], cos, sin, f, c["interleaved"])[:n].to(torch.bfloat16)
    if c["k_out"]:
        s["k_rows"][:n] = k.to(torch.bfloat16)
    v, slot = s["v"][:n].float(), s["slot_map"][:n]
    if c["fp8"]:
        k = (k / s["k_scale"][:, None]).clamp(-448, 448)
        v = (v / s["v_scale"][:, None]).clamp(-448, 448)
    # (the codes of an FP8 pool are moved as bytes: index assignment does not take them)
    as_stored = (lambda x: x.to(torch.float8_e4m3fn).view(torch.uint8)) if c["fp8"] else \
        (lambda x: x.to(torch.bfloat16))
    seen = (lambda p: p.view(torch.uint8).view(-1, c["hkv"], D)) if c["fp8"] else (lambda p: p.view(-1, c["hkv"], D))
    seen(s["k_pages"])[slot] = as_stored(k)
    seen(s["v_pages"])[slot] = as_stored(v)
    return _rope_answer(s)


def _prefill_answer(s):
    return {"out": s["out"], "lse": s["lse"]} if s["lse"] is not None else {"out": s["out"]}


def _run_prefill(s):
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        ra.prefill(s["q"], s["k"], s["v"], s["indptr"], s["scale"], out=s["out"], lse=s["lse"])
        return _prefill_answer(s)
    # the prompts padded to the longest: query rows of a KV head beside each other, one product for each prompt and head
    c, n, real = s["case"], s["longest"], s["real"]
    batch, hq, hkv = c["batch"], c["hq"], c["hkv"]
    group = hq // hkv
    start = s["indptr"][:-1].long()
    lens = s["indptr"][1:].long() - start
    at = torch.arange(n, device=DEVICE)
    rows = (start[:, None] + at).clamp(max=max(real - 1, 0))
    q = s["q"][rows].float().view(batch, n, hkv, group, D).permute(0, 2, 3, 1, 4).reshape(batch, hkv, group * n, D)
    k = s["k"][rows].float().permute(0, 2, 3, 1).contiguous()
    v = s["v"][rows].float().permute(0, 2, 1, 3).contiguous()
    x = torch.matmul(q * s["scale"], k).view(batch, hkv, group, n, n)
    x.masked_fill_(at[None, :] > at[:, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(batch, hkv, group * n, n), v).view(batch, hkv, group, n, D) / total
    b = torch.repeat_interleave(torch.arange(batch, device=DEVICE), lens, output_size=real)
    i = torch.arange(real, device=DEVICE) - start[b]
    s["out"][:real] = o.permute(0, 3, 1, 2, 4).reshape(batch, n, hq, D)[b, i].to(torch.bfloat16)
    if s["lse"] is not None:
        lse = (top + total.log()).squeeze(-1)
        s["lse"][:real] = lse.permute(0, 3, 1, 2).reshape(batch, n, hq)[b, i]
    return _prefill_answer(s)


# ------------------------------------------------------------------------------------------------------- work

def work(case):
    c = _full(case)
    if c["op"] == "map":
        cached, new = _lens(c, c["cached_lo"], c["cached_hi"], 1), _lens(c, c["new_lo"], c["new_hi"], 2)
        pages = int((-(-(cached + new) // c["page"]) - -(-cached // c["page"])).sum())
        rows = int(new.sum()) + c["pad"]
        return {"bytes": c["batch"] * (20 if c["delta"] else 16) + 12 * rows + 8 * pages + 12, "flops": 0}
    if c["op"] == "prefill":
        n = _lens(c, c["len_lo"], c["len_hi"]).astype(np.float64)
        rows = float(n.sum())
        return {"bytes": rows * (2 * c["hq"] + 2 * c["hkv"]) * 2 * D + (rows * c["hq"] * 4 if c["lse"] else 0)
                + 4 * (c["batch"] + 1), "flops": float((n * (n + 1) / 2).sum()) * 4 * D * c["hq"]}
    hq, hkv, rows = c["hq"], c["hkv"], c["rows"]
    read, write = hq + hkv, hq + hkv                     # heads of 2 D bytes, for each row
    if c["op"] == "rope_append":
        read += hkv
        write = hq + (hkv if c["k_out"] else 0) + 2 * hkv * (0.5 if c["fp8"] else 1.0)
    axes = 3 if c["axes"] else 1
    return {"bytes": rows * ((read + write) * 2 * D + 4 * axes + (8 if c["op"] == "rope_append" else 0)),
            "flops": rows * (hq + hkv) * c["rotated"] * 3.0}


# ------------------------------------------------------------------------------------------------------ exact

def exact(case, seed):
    c = _full(case)
    if c["op"] == "map":
        return None                                      # whole numbers only
    s = prepare(case, seed)
    return _exact_prefill(c, s) if c["op"] == "prefill" else _exact_rope(c, s)


def _exact_turned(x, pos, freq, which, sign, interleaved):
    """Each pair as a complex number, multiplied by exp(i theta)."""
    f = freq.shape[0]
    x = x.double().clone()
    lo = torch.arange(f, device=DEVICE) * 2 if interleaved else torch.arange(f, device=DEVICE)
    hi = lo + 1 if interleaved else lo + f
    theta = sign * freq.double()[None, :] * pos.double().T.gather(1, which[None, :].expand(pos.shape[1], -1))
    turn = torch.polar(torch.ones_like(theta), theta)[:, None, :]
    z = torch.complex(x[..., lo], x[..., hi]) * turn
    x[..., lo], x[..., hi] = z.real, z.imag
    return x


def _exact_rope(c, s):
    n = c["rows"]
    which = torch.zeros(s["inv_freq"].shape[0], dtype=torch.long, device=DEVICE) if s["axes"] is None else \
        s["axes"].long()
    sign = -1.0 if c["inverse"] else 1.0
    q, k = (_exact_turned(s[name], s["positions"], s["inv_freq"], which, sign, c["interleaved"]) for name in "qk")
    q[n:], k[n:] = 0, 0
    if c["op"] == "rope":
        return {"q": q, "k": k}
    out = {"q": q}
    for name, rows, scale in (("k_pages", k, s["k_scale"]), ("v_pages", s["v"].double(), s["v_scale"])):
        pool = torch.zeros(s[name].shape, dtype=torch.float64, device=DEVICE)
        x = rows[:n]
        if c["fp8"]:
            x = (x / scale.double()[:, None]).clamp(-448, 448)
        pool.view(-1, c["hkv"], D)[s["slot_map"][:n]] = x
        out[name] = pool
    return {**out, "k": k} if c["k_out"] else out


def _exact_prefill(c, s):
    hq, hkv = c["hq"], c["hkv"]
    rows = s["q"].shape[0]
    out = torch.zeros((rows, hq, D), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((rows, hq), dtype=torch.float64, device=DEVICE)
    ends = s["indptr"].tolist()
    for lo, hi in zip(ends[:-1], ends[1:]):
        for g in range(hkv):
            heads = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            k, v = s["k"][lo:hi, g].double(), s["v"][lo:hi, g].double()
            for r in range(lo, hi, 1024):
                e = min(hi, r + 1024)
                q = s["q"][r:e, heads].double().transpose(0, 1)
                x = s["scale"] * (q @ k[:e - lo].T)
                seen = torch.arange(e - lo, device=DEVICE)[None, :] <= torch.arange(r - lo, e - lo, device=DEVICE)[:, None]
                z = torch.where(seen, x, -math.inf)
                each = torch.logsumexp(z, dim=-1)
                out[r:e, heads] = (torch.exp(z - each[..., None]) @ v[:e - lo]).transpose(0, 1)
                lse[r:e, heads] = each.T
    return {"out": out, "lse": lse} if s["lse"] is not None else {"out": out}
