"""What the speed of the operators at a step's ends is measured on: normed rotary rows with their append and their
gradient, log probabilities of tokens with their gradient, requests that fork and drop their tokens.

A case is one use of the public entry points of ``paper_2609_08368_amd.rl_attn``. ``op`` names it:

* "norm_append": queries and keys normed and rotated in one pass with the append of a step's rows to their pages
  (``norm_rope_append_kv`` or, with ``fp8``, ``norm_rope_append_kv_fp8``);
* "norm_train": the same rows without pages, and their gradient (``norm_rope``, ``norm_rope_backward``);
* "logprobs": log probabilities of given tokens, entropies and the likeliest alternatives (``token_logprobs``);
* "logprobs_train": the same without alternatives, and the gradient of the logits (``token_logprobs_backward``);
* "fork": requests that begin as copies of others, and the copies of their last pages in every layer
  (``fork_requests``, ``copy_pages``);
* "drop": requests that end or are cut back, and the pages this frees (``drop_tokens``).

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
EPS = 1e-6                       # of the norms
MOST_LOGITS = 4096 * 131072      # bytes of the largest logits / 2
MOST_HEADS = 16384 * 72          # (row, head) pairs of the largest normed call with its gradient
MOST_TABLE = 1 << 21             # entries of the largest block table
MOST_POOL = 16 * 4096 * 8 * 4    # (token, head, layer) triples of the largest fork's prompts
MOST_COPIED = 128 * 64 * 8 * 4   # (token, head, layer) triples of its copies

# every field a case may leave out
DEFAULTS = {
    "pad": 0,                    # norm_append: rows behind the last request's (a batch padded to a captured size)
    "fp8": False,                # E4M3 pages (norm_append: with one scale per KV head)
    "k_out": False,              # norm_append: the keys are wanted as rows too
    "axes": "",                  # "" one axis, "blocks" or "cycle": three, by blocks of frequencies or in turn
    "rotated": D,                # dimensions that are rotated
    "interleaved": False,        # pairs of neighbours instead of halves
    "far": 0,                    # positions start here
    "page": 64,
    "weights_f32": False,        # norm weights in fp32 instead of bf16
    "f32": False,                # logits in fp32 instead of bf16
    "top": 0,                    # alternatives asked for
    "scaled": False,             # each row has a scale (an inverse temperature) of its own
    "masked": 0.0,               # share of the rows without a token (prompts, padding)
    "stride_pad": 0,             # columns of the logits' buffer behind the vocabulary
    "banned": False,             # some rows have most of their tokens excluded (-inf)
}


def listed():
    return [
        # a decode step of the 128 agentic sessions on a 96/8-head model with normed heads, text beside images
        {"name": "norm_append_decode", "op": "norm_append", "rows": 128, "hq": 96, "hkv": 8, "axes": "blocks",
         "far": 60000, "shape_seed": 1},
        # an odd number of turns' rows into an FP8 cache, whose keys are wanted as rows too, padded
        {"name": "norm_append_fp8", "op": "norm_append", "rows": 20011, "hq": 64, "hkv": 8, "fp8": True, "k_out": True,
         "pad": 213, "shape_seed": 2},
        # training: the rows of a packed batch of 16K tokens and their gradient
        {"name": "norm_train", "op": "norm_train", "rows": 16384, "hq": 64, "hkv": 8, "shape_seed": 3},
        # training a small model, half of each head rotated, pairs of neighbours, fp32 weights
        {"name": "norm_train_small", "op": "norm_train", "rows": 1777, "hq": 8, "hkv": 2, "rotated": 64,
         "interleaved": True, "weights_f32": True, "shape_seed": 4},
        # one token of one session, fp32 logits, five alternatives: latency
        {"name": "logprobs_one", "op": "logprobs", "rows": 1, "vocab": 32000, "f32": True, "top": 5, "shape_seed": 5},
        # a decode step of the 128 sessions: 20 alternatives, a temperature each, some held to a grammar
        {"name": "logprobs_decode", "op": "logprobs", "rows": 128, "vocab": 131072, "top": 20, "scaled": True,
         "banned": True, "shape_seed": 6},
        # training on a packed batch: 4096 tokens, a third of them prompts that the loss leaves out
        {"name": "logprobs_train", "op": "logprobs_train", "rows": 4096, "vocab": 131072, "masked": 0.3,
         "shape_seed": 7},
        # an odd vocabulary in fp32, rows that start at any multiple of four bytes
        {"name": "logprobs_train_odd", "op": "logprobs_train", "rows": 701, "vocab": 50021, "f32": True,
         "stride_pad": 2, "scaled": True, "shape_seed": 8},
        # one group of eight attempts begins from its prompt, one layer: latency
        {"name": "fork_group", "op": "fork", "parents": 1, "attempts": 8, "len_lo": 1111, "len_hi": 1111, "hkv": 8,
         "layers": 1, "shape_seed": 9},
        # 16 groups of eight begin from prompts of up to 4096 tokens, four layers
        {"name": "fork_groups", "op": "fork", "parents": 16, "attempts": 8, "len_lo": 2000, "len_hi": 4096, "hkv": 8,
         "layers": 4, "shape_seed": 10},
        # between steps of the 128 sessions in 16 groups: some end, some are cut back to an earlier turn
        {"name": "drop_sessions", "op": "drop", "groups": 16, "attempts": 8, "prompt": 4096, "len_hi": 65536,
         "shape_seed": 11},
        # many short requests in small pages
        {"name": "drop_many", "op": "drop", "groups": 750, "attempts": 4, "prompt": 160, "len_hi": 901, "page": 16,
         "shape_seed": 12},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any mix of heads, formats and options, sizes over the logarithm of their range."""
    op = rng.choice(["norm_append", "norm_append", "norm_train", "logprobs", "logprobs", "logprobs_train", "fork",
                     "drop"])
    c = {"op": op, "shape_seed": rng.randrange(1 << 20)}
    page = rng.choice([8, 16, 32, 64, 64, 128])
    if op in ("norm_append", "norm_train"):
        hq, hkv = rng.choice([(8, 2), (32, 8), (64, 8), (64, 8), (96, 8), (16, 16), (8, 1), (12, 1)])
        c.update(rows=_log_int(rng, 1, min(65536, MOST_HEADS // (hq + 3 * hkv))), hq=hq, hkv=hkv,
                 axes=rng.choice(["", "blocks", "cycle"]), rotated=rng.choice([D, D, 96, 64, 32]),
                 interleaved=rng.random() < 0.3, far=rng.choice([0, _log_int(rng, 100, 1 << 20)]),
                 weights_f32=rng.random() < 0.3)
        if op == "norm_append":
            c.update(page=page, fp8=rng.random() < 0.4, k_out=rng.random() < 0.4,
                     pad=rng.choice([0, 0, rng.randrange(1, 300)]))
    elif op in ("logprobs", "logprobs_train"):
        f32 = rng.random() < 0.3
        vocab = _log_int(rng, 500, 262144)
        rows = _log_int(rng, 1, min(16384, MOST_LOGITS // vocab // (2 if f32 else 1)))
        c.update(vocab=vocab, rows=rows, f32=f32, scaled=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.4]),
                 stride_pad=rng.choice([0, 0, rng.randrange(1, 64)]), banned=rng.random() < 0.3)
        if op == "logprobs":
            c["top"] = rng.choice([0, 1, 5, 20, 32])
    elif op == "fork":
        parents, attempts = _log_int(rng, 1, 128), rng.choice([1, 2, 8, 8, 16])
        hkv, layers = rng.choice([1, 2, 8]), rng.choice([1, 2, 4])
        parents = max(1, min(parents, MOST_COPIED // (attempts * page * hkv * layers)))
        hi = min(_log_int(rng, 1, 8192), MOST_TABLE // (parents * (attempts + 1)) * page,
                 MOST_POOL // (parents * hkv * layers))
        c.update(parents=parents, attempts=attempts, hkv=hkv, layers=layers, len_lo=rng.choice([0, hi // 2, hi]),
                 len_hi=hi, page=page, fp8=rng.random() < 0.4)
    else:
        groups, attempts = _log_int(rng, 1, 512), rng.choice([1, 4, 8])
        hi = min(_log_int(rng, 1, 65536), MOST_TABLE // (groups * attempts) * page)
        c.update(groups=groups, attempts=attempts, len_hi=hi, prompt=rng.choice([0, hi // 4, hi // 2]), page=page)
    return c


def _full(case):
    return {**DEFAULTS, **case}


def _dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device=DEVICE, dtype=dtype)


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(seed, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_gen(seed), device=DEVICE).to(dtype)


# ------------------------------------------------------------------------------------------------ preparation

def prepare(case, seed):
    c = _full(case)
    s = {"case": c}
    {"norm_append": _prepare_norm, "norm_train": _prepare_norm, "logprobs": _prepare_logprobs,
     "logprobs_train": _prepare_logprobs, "fork": _prepare_fork, "drop": _prepare_drop}[c["op"]](c, seed, s)
    return s


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


def _prepare_norm(c, seed, s):
    rng = np.random.default_rng(seed + 1)
    rows, hq, hkv, page = c["rows"] + c["pad"], c["hq"], c["hkv"], c["page"]
    f = c["rotated"] // 2
    qkv = _normal(seed, (rows, hq + 2 * hkv, D))         # as a fused projection leaves them
    qkv *= _dev(rng.uniform(0.2, 5.0, hq + 2 * hkv), torch.bfloat16)[None, :, None]   # heads of different size
    axis = {"": None, "blocks": np.repeat([0, 1, 2], [f - 2 * (3 * f // 8), 3 * f // 8, 3 * f // 8]),
            "cycle": np.arange(f) % 3}[c["axes"]]
    kind = torch.float32 if c["weights_f32"] else torch.bfloat16
    s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], real=c["rows"],
             q_weight=_dev(rng.uniform(0.3, 2.0, D), kind), k_weight=_dev(rng.uniform(0.3, 2.0, D), kind),
             positions=_dev(_positions(c, seed + 2, rows).reshape(-1, rows), torch.int32),
             inv_freq=_dev(1e6 ** (-np.arange(f) / f), torch.float32),
             axes=None if axis is None else _dev(axis, torch.int32),
             q_out=torch.zeros((rows, hq, D), dtype=torch.bfloat16, device=DEVICE),
             k_rows=torch.zeros((rows, hkv, D), dtype=torch.bfloat16, device=DEVICE))
    if c["op"] == "norm_train":
        s.update(dq_out=_normal(seed + 3, (rows, hq, D)), dk_out=_normal(seed + 4, (rows, hkv, D)),
                 dq=torch.zeros((rows, hq, D), dtype=torch.bfloat16, device=DEVICE),
                 dk=torch.zeros((rows, hkv, D), dtype=torch.bfloat16, device=DEVICE),
                 dq_weight=torch.zeros(D, device=DEVICE), dk_weight=torch.zeros(D, device=DEVICE))
        return
    pool = -(-c["rows"] // page) + 7
    order = rng.permutation(pool)
    at = np.arange(c["rows"]) + int(rng.integers(0, page))
    slots = np.concatenate([order[at // page] * page + at % page, np.full(c["pad"], -1)])
    kind = torch.float8_e4m3fn if c["fp8"] else torch.bfloat16
    s.update(slot_map=_dev(slots, torch.int64),
             k_pages=torch.zeros((pool, page, hkv, D), dtype=kind, device=DEVICE),
             v_pages=torch.zeros((pool, page, hkv, D), dtype=kind, device=DEVICE),
             k_scale=_dev(rng.uniform(0.02, 0.04, hkv), torch.float32),
             v_scale=_dev(rng.uniform(0.03, 0.06, hkv), torch.float32))


def _prepare_logprobs(c, seed, s):
    rng = np.random.default_rng(seed + 1)
    rows, vocab, k = c["rows"], c["vocab"], c["top"]
    kind = torch.float32 if c["f32"] else torch.bfloat16
    x = torch.empty((rows, vocab + c["stride_pad"]), dtype=kind, device=DEVICE)
    g = _gen(seed)
    sharp = _dev(rng.uniform(0.5, 4.0, rows), torch.float32)       # rows of a sure and an unsure model
    tokens = torch.empty(rows, dtype=torch.int64, device=DEVICE)
    for lo in range(0, rows, 512):
        y = torch.randn((min(rows, lo + 512) - lo, x.shape[1]), generator=g, device=DEVICE) * sharp[lo:lo + 512, None]
        y = y.to(kind)
        if c["banned"]:                                  # a grammar leaves one token in 97
            y[::3, torch.arange(x.shape[1], device=DEVICE) % 97 != 5] = -math.inf
        x[lo:lo + 512] = y
        # a token that the row might have been sampled to
        u = torch.rand(y.shape[0], vocab, generator=g, device=DEVICE)
        tokens[lo:lo + 512] = (y[:, :vocab].float() - torch.log(-torch.log(u.clamp(1e-30, 1 - 1e-7)))).argmax(-1)
    if c["masked"]:
        tokens[_dev(rng.random(rows) < c["masked"], torch.bool)] = -1
    s.update(logits=x[:, :vocab], tokens=tokens,
             row_scale=_dev(rng.uniform(0.7, 1.5, rows), torch.float32) if c["scaled"] else None,
             logprobs=torch.zeros(rows, device=DEVICE), entropy=torch.zeros(rows, device=DEVICE),
             lse=torch.zeros(rows, device=DEVICE))
    if k:
        s.update(top_ids=torch.zeros((rows, k), dtype=torch.int32, device=DEVICE),
                 top_logprobs=torch.zeros((rows, k), device=DEVICE))
    if c["op"] == "logprobs_train":
        s.update(d_logprobs=_dev(rng.standard_normal(rows), torch.float32),
                 d_entropy=_dev(rng.standard_normal(rows) * 0.1, torch.float32),
                 d_logits=torch.zeros((rows, vocab), dtype=kind, device=DEVICE))


def _prepare_fork(c, seed, s):
    """Rows of the table: the cached prompts, and behind them the attempts that begin, in a shuffled order."""
    rng, shape = np.random.default_rng(seed), np.random.default_rng(c["shape_seed"])
    page, n, each = c["page"], c["parents"], c["attempts"]
    batch = n * (each + 1)
    plen = shape.integers(c["len_lo"], c["len_hi"] + 1, n)
    back = shape.integers(0, 1 + np.minimum(plen, 7)) * (shape.random(n) < 0.3)   # some begin before the prompt's end
    where = shape.permutation(batch)
    parent_row, child_row = where[:n], where[n:]
    parents, lens, fork_lens = np.full(batch, -1), np.zeros(batch, np.int64), np.zeros(batch, np.int64)
    lens[parent_row] = plen
    parents[child_row] = np.repeat(parent_row, each)
    fork_lens[child_row] = np.repeat(plen - back, each)
    held = -(-lens // page)
    width = int(held.max()) + 3
    pool = int(held.sum()) + n * each + 40
    ids = rng.permutation(pool)
    table = np.full((batch, width), -1, np.int64)
    table[np.arange(width)[None] < held[:, None]] = ids[:int(held.sum())]
    used = int(rng.integers(0, 40))
    free = np.concatenate([rng.integers(0, pool, used), ids[int(held.sum()):]])
    kind = torch.float8_e4m3fn if c["fp8"] else torch.bfloat16
    s.update(parents=_dev(parents, torch.int32), fork_lens=_dev(fork_lens, torch.int32), kv_lens=_dev(lens, torch.int32),
             free_pages=_dev(free, torch.int32), free_used=_dev(np.array([used]), torch.int32),
             block_table=_dev(table, torch.int32), pages=pool, moved=int((fork_lens % page).sum()),
             kv_out=torch.zeros(batch, dtype=torch.int32, device=DEVICE),
             used_out=torch.zeros(1, dtype=torch.int32, device=DEVICE),
             copies=torch.zeros((batch, 3), dtype=torch.int32, device=DEVICE),
             pools=[tuple(_normal(seed + 2 * i + j, (pool, page, c["hkv"], D)).to(kind) for j in (0, 1))
                    for i in range(c["layers"])])


def _drop_lens(c):
    """Lengths now and to be kept: a fifth of the requests ends, a fifth is cut back by up to a turn."""
    shape = np.random.default_rng(c["shape_seed"])
    batch = c["groups"] * c["attempts"]
    # most sessions are far from the longest
    lens = c["prompt"] + ((c["len_hi"] - c["prompt"]) * shape.random(batch) ** 2).astype(np.int64)
    lens[int(shape.integers(batch))] = c["len_hi"]
    what = shape.random(batch)
    keep = np.where(what < 0.2, 0, np.where(what < 0.4, lens - shape.integers(1, 2048, batch), lens))
    return lens, np.maximum(keep, np.where(keep > 0, c["prompt"], 0))


def _prepare_drop(c, seed, s):
    rng = np.random.default_rng(seed)
    page, each = c["page"], c["attempts"]
    lens, keep = _drop_lens(c)
    batch = len(lens)
    held, shared = -(-lens // page), c["prompt"] // page           # whole pages of the prompt are shared
    width = int(held.max()) + 3
    own_pages = np.maximum(held - shared, 0)
    pool = c["groups"] * shared + int(own_pages.sum()) + 50
    ids = rng.permutation(pool)
    table = np.full((batch, width), -1, np.int64)
    j = np.arange(width)[None]
    table[:, :shared] = np.repeat(ids[:c["groups"] * shared].reshape(c["groups"], shared), each, axis=0)
    table[(j >= shared) & (j < held[:, None])] = ids[c["groups"] * shared:pool - 50]
    free = np.concatenate([rng.integers(0, pool, pool - 50), ids[pool - 50:]])    # the taken entries are stale
    s.update(kv_lens=_dev(lens, torch.int32), keep_lens=_dev(keep, torch.int32), block_table=_dev(table, torch.int32),
             free_pages=_dev(free, torch.int32), free_used=_dev(np.array([pool - 50]), torch.int32), pages=pool,
             kv_out=torch.zeros(batch, dtype=torch.int32, device=DEVICE),
             used_out=torch.zeros(1, dtype=torch.int32, device=DEVICE))


# ------------------------------------------------------------------------------------------------------- runs

def run(state):
    return {"norm_append": _run_norm_append, "norm_train": _run_norm_train, "logprobs": _run_logprobs,
            "logprobs_train": _run_logprobs, "fork": _run_fork, "drop": _run_drop}[state["case"]["op"]](state)


def _angles(s):
    """cos and sin [rows, 1, F] of position times frequency: the angle in 64 bits, where far positions need them."""
    pos = s["positions"].double()
    which = s["axes"].long() if s["axes"] is not None else torch.zeros(s["inv_freq"].shape[0], dtype=torch.long,
                                                                       device=DEVICE)
    a = pos[which].T * s["inv_freq"].double()
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _rotate(x, cos, sin, f, interleaved):
    if interleaved:
        a, b = x[..., 0:2 * f:2], x[..., 1:2 * f:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :f], x[..., f:2 * f]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, x[..., 2 * f:]), dim=-1)


def _normed(x):
    """A head's row over its root mean square, and one over that."""
    x = x.float()
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    return x * r, r


def _norm_answer(s):
    out = {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    return {**out, "k": s["k_rows"]} if s["case"]["k_out"] else out


def _run_norm_append(s):
    c = s["case"]
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        k_out = s["k_rows"] if c["k_out"] else None
        if c["fp8"]:
            ra.norm_rope_append_kv_fp8(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], EPS, s["positions"],
                                       s["inv_freq"], s["slot_map"], s["k_pages"], s["v_pages"], s["k_scale"],
                                       s["v_scale"], s["axes"], interleaved=c["interleaved"], q_out=s["q_out"],
                                       k_out=k_out)
        else:
            ra.norm_rope_append_kv(s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], EPS, s["positions"],
                                   s["inv_freq"], s["slot_map"], s["k_pages"], s["v_pages"], s["axes"],
                                   interleaved=c["interleaved"], q_out=s["q_out"], k_out=k_out)
        return _norm_answer(s)
    n, f = s["real"], s["inv_freq"].shape[0]
    cos, sin = (x[:n] for x in _angles(s))
    q = _rotate(_normed(s["q"][:n])[0] * s["q_weight"].float(), cos, sin, f, c["interleaved"])
    k = _rotate(_normed(s["k"][:n])[0] * s["k_weight"].float(), cos, sin, f, c["interleaved"])
    s["q_out"][:n] = q.to(torch.bfloat16)
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
    return _norm_answer(s)


def _run_norm_train(s):
    c = s["case"]
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        ra.norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], EPS, s["positions"], s["inv_freq"], s["axes"],
                     interleaved=c["interleaved"], q_out=s["q_out"], k_out=s["k_rows"])
        ra.norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["q_weight"], s["k_weight"], EPS,
                              s["positions"], s["inv_freq"], s["axes"], interleaved=c["interleaved"], dq=s["dq"],
                              dk=s["dk"], dq_weight=s["dq_weight"], dk_weight=s["dk_weight"])
    else:
        f = s["inv_freq"].shape[0]
        cos, sin = _angles(s)
        for x, w, out, d_out, dx, dw in (("q", "q_weight", "q_out", "dq_out", "dq", "dq_weight"),
                                         ("k", "k_weight", "k_rows", "dk_out", "dk", "dk_weight")):
            y, r = _normed(s[x])
            weight = s[w].float()
            s[out].copy_(_rotate(y * weight, cos, sin, f, c["interleaved"]))
            g = _rotate(s[d_out].float(), cos, -sin, f, c["interleaved"])
            s[dw].copy_((g * y).sum(dim=(0, 1)))
            u = g * weight
            s[dx].copy_(r * (u - y * (u * y).mean(dim=-1, keepdim=True)))
    return {"q": s["q_out"], "k": s["k_rows"], "dq": s["dq"], "dk": s["dk"], "dq_weight": s["dq_weight"],
            "dk_weight": s["dk_weight"]}


def _logprobs_answer(s):
    out = {k: s[k] for k in ("logprobs", "entropy", "lse")}
    if s["case"]["top"]:
        out.update(top_ids=s["top_ids"], top_logprobs=s["top_logprobs"])
    if s["case"]["op"] == "logprobs_train":
        out["d_logits"] = s["d_logits"]
    return out


def _run_logprobs(s):
    c = s["case"]
    train = c["op"] == "logprobs_train"
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        top = {"top_ids": s["top_ids"], "top_logprobs": s["top_logprobs"]} if c["top"] else {}
        ra.token_logprobs(s["logits"], s["tokens"], s["row_scale"], logprobs=s["logprobs"], entropy=s["entropy"],
                          lse=s["lse"], **top)
        if train:
            ra.token_logprobs_backward(s["logits"], s["tokens"], s["lse"], s["d_logprobs"], s["row_scale"],
                                       entropy=s["entropy"], d_entropy=s["d_entropy"], d_logits=s["d_logits"])
        return _logprobs_answer(s)
    has = s["tokens"] >= 0                               # rows without a token: zeros, no alternatives
    scale = s["row_scale"][:, None] if s["row_scale"] is not None else 1.0
    at = s["tokens"].clamp(min=0)[:, None]
    z = s["logits"].float() * scale
    top = z.amax(dim=-1, keepdim=True)
    z -= top
    e = z.exp()
    total = e.sum(dim=-1, keepdim=True)
    log_total = total.log()
    log_p = z.sub_(log_total)
    p = e.div_(total)
    finite = log_p.clamp(min=-1e30)                      # (an excluded token adds nothing)
    entropy = -(p * finite).sum(dim=-1)
    s["logprobs"].copy_(log_p.gather(1, at)[:, 0].where(has, 0.0))
    s["entropy"].copy_(entropy.where(has, 0.0))
    s["lse"].copy_((top + log_total)[:, 0].where(has, 0.0))
    if c["top"]:
        # unique keys: the logit's order, then the lower index
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits)
        key = (key << 32) + (c["vocab"] - torch.arange(c["vocab"], device=DEVICE))
        ids = c["vocab"] - (key.topk(c["top"], dim=-1).values & 0xffffffff)
        lp = log_p.gather(1, ids)
        real = has[:, None] & (lp > -math.inf)
        s["top_ids"].copy_(ids.where(real, -1))
        s["top_logprobs"].copy_(lp.where(real, -math.inf))
    if train:
        g, h = s["d_logprobs"].where(has, 0.0)[:, None], s["d_entropy"].where(has, 0.0)[:, None]
        d = p * -(g + h * (finite + entropy[:, None]))
        d.scatter_add_(1, at, g)
        s["d_logits"].copy_(d.mul_(scale))
    return _logprobs_answer(s)


def _run_fork(s):
    page = s["case"]["page"]
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        ra.fork_requests(s["parents"], s["fork_lens"], s["kv_lens"], s["free_pages"], s["free_used"], s["block_table"],
                         page, s["pages"], kv_lens_out=s["kv_out"], free_used_out=s["used_out"], copies=s["copies"])
        for k, v in s["pools"]:
            ra.copy_pages(s["copies"], k, v)
    else:
        forked = s["parents"] >= 0
        parent, n = s["parents"].long().clamp(min=0), s["fork_lens"].long()
        full, rest = n // page, n % page
        need = forked & (rest > 0)
        fresh = s["free_pages"][(s["free_used"] + need.long().cumsum(0) - 1).clamp(0, s["free_pages"].shape[0] - 1)]
        width = s["block_table"].shape[1]
        j = torch.arange(width, device=DEVICE)
        theirs = s["block_table"][parent]
        shared = forked[:, None] & (j < full[:, None])
        last = need[:, None] & (j == full[:, None])
        source = theirs.gather(1, full.clamp(max=width - 1)[:, None])[:, 0]
        s["block_table"].copy_(torch.where(shared, theirs, torch.where(last, fresh[:, None], s["block_table"])))
        s["kv_out"].copy_(torch.where(forked, s["fork_lens"], s["kv_lens"]))
        s["used_out"].copy_(s["free_used"] + need.sum())
        s["copies"].copy_(torch.stack((source.where(need, -1), fresh.where(need, -1), rest.where(need, 0)), dim=-1))
        # the copied rows one by one
        each = torch.repeat_interleave(torch.arange(len(rest), device=DEVICE), s["copies"][:, 2],
                                       output_size=s["moved"])
        row = torch.arange(s["moved"], device=DEVICE) - (s["copies"][:, 2].cumsum(0) - s["copies"][:, 2])[each]
        src, dst = (s["copies"][each, i].long() * page + row for i in (0, 1))
        for pool in s["pools"]:
            for x in pool:
                # (E4M3 codes are moved as bytes: index assignment does not take them)
                flat = (x.view(torch.uint8) if s["case"]["fp8"] else x).view(-1, x.shape[2], D)
                flat[dst] = flat[src]
    return {"block_table": s["block_table"], "kv_lens": s["kv_out"], "free_used": s["used_out"], "copies": s["copies"],
            "pools": [x for pool in s["pools"] for x in pool]}


def _run_drop(s):
    page = s["case"]["page"]
    if own:
        from paper_2609_08368_amd import rl_attn as ra

        ra.drop_tokens(s["kv_lens"], s["keep_lens"], s["block_table"], s["free_pages"], s["free_used"], page,
                       s["pages"], kv_lens_out=s["kv_out"], free_used_out=s["used_out"])
    else:
        kept = torch.minimum(s["kv_lens"], s["keep_lens"])
        before, after = (s["kv_lens"] + page - 1) // page, (kept + page - 1) // page
        j = torch.arange(s["block_table"].shape[1], device=DEVICE)[None]
        mark = torch.zeros((2, s["pages"] + 1), dtype=torch.bool, device=DEVICE)
        for i, inside in enumerate((j < after[:, None], (j >= after[:, None]) & (j < before[:, None]))):
            mark[i, torch.where(inside, s["block_table"], s["pages"]).long().flatten()] = True
        freed = (mark[1] & ~mark[0])[:-1]
        n = freed.sum()
        rank = freed.long().cumsum(0) - 1
        entries = s["free_pages"].shape[0]
        at = torch.where(freed, s["free_used"] - n + rank, entries)
        grown = torch.cat((s["free_pages"], s["free_pages"][:1]))
        grown[at] = torch.arange(s["pages"], dtype=torch.int32, device=DEVICE)
        s["free_pages"].copy_(grown[:-1])
        s["kv_out"].copy_(kept)
        s["used_out"].copy_(s["free_used"] - n)
    return {"free_pages": s["free_pages"], "kv_lens": s["kv_out"], "free_used": s["used_out"]}


# ------------------------------------------------------------------------------------------------------- work

def work(case):
    c = _full(case)
    op = c["op"]
    if op in ("logprobs", "logprobs_train"):
        size = 4 if c["f32"] else 2
        rows = c["rows"] * (1 - c["masked"])             # the logits of rows without a token need not be read
        n = rows * c["vocab"]
        each = 8 + 12 + 8 * c["top"] + (4 if c["scaled"] else 0)
        if op == "logprobs":
            return {"bytes": n * size + c["rows"] * each, "flops": n * 5.0}
        return {"bytes": 2 * n * size + c["rows"] * (c["vocab"] * size + 2 * each), "flops": n * 12.0}
    if op == "fork":
        s = np.random.default_rng(c["shape_seed"])
        plen = s.integers(c["len_lo"], c["len_hi"] + 1, c["parents"])
        kept = plen - s.integers(0, 1 + np.minimum(plen, 7)) * (s.random(c["parents"]) < 0.3)
        rows = float((kept % c["page"]).sum())
        # the attempts' rows of a group come from one source
        moved = (rows + rows * c["attempts"]) * 2 * c["layers"] * c["hkv"] * D * (1 if c["fp8"] else 2)
        entries = float((-(-kept // c["page"])).sum())
        return {"bytes": moved + 4 * entries * (1 + c["attempts"]) + c["parents"] * (c["attempts"] + 1) * 28.0 + 8,
                "flops": 0}
    if op == "drop":
        lens, _ = _drop_lens(c)
        return {"bytes": 4.0 * float((-(-lens // c["page"])).sum()) + 12.0 * len(lens) + 8, "flops": 0}
    rows, hq, hkv = c["rows"], c["hq"], c["hkv"]
    axes = 3 if c["axes"] else 1
    pairs = rows * (hq + hkv)
    if op == "norm_train":
        # forward reads and writes a head row; its gradient reads that row and the outputs' gradient and writes one
        return {"bytes": pairs * 2.0 * D * 5 + rows * 8.0 * axes, "flops": pairs * D * 20.0}
    moved = hq + 2 * hkv + hq + (hkv if c["k_out"] else 0) + 2 * hkv * (0.5 if c["fp8"] else 1.0)
    return {"bytes": rows * (moved * 2 * D + 4 * axes + 8.0), "flops": pairs * D * 7.0}


# ------------------------------------------------------------------------------------------------------ exact

def exact(case, seed):
    c = _full(case)
    if c["op"] in ("fork", "drop"):
        return None                                      # whole numbers and copies only
    s = prepare(case, seed)
    return _exact_logprobs(c, s) if c["op"].startswith("logprobs") else _exact_norm(c, s)


def _turns(s, dtype):
    """exp(i angle) of every row and frequency."""
    f = s["inv_freq"].shape[0]
    which = torch.zeros(f, dtype=torch.long, device=DEVICE) if s["axes"] is None else s["axes"].long()
    theta = s["inv_freq"].double()[None, :] * s["positions"].double().T.gather(
        1, which[None, :].expand(s["positions"].shape[1], -1))
    return torch.polar(torch.ones_like(theta), theta)[:, None, :].to(dtype)


def _exact_turned(x, turn, interleaved):
    x = x.clone()
    f = turn.shape[-1]
    lo = torch.arange(f, device=DEVICE) * 2 if interleaved else torch.arange(f, device=DEVICE)
    hi = lo + 1 if interleaved else lo + f
    z = torch.complex(x[..., lo], x[..., hi]) * turn
    x[..., lo], x[..., hi] = z.real, z.imag
    return x


def _exact_norm(c, s):
    n = c["rows"]
    turn = _turns(s, torch.complex128)
    out = {}
    for name, d_out in (("q", "dq_out"), ("k", "dk_out")):
        w = s[name + "_weight"].double()
        y = torch.zeros(s[name].shape, dtype=torch.float64, device=DEVICE)
        dx = torch.zeros_like(y) if c["op"] == "norm_train" else None
        dw = torch.zeros(D, dtype=torch.float64, device=DEVICE)
        for lo in range(0, n, 2048):
            rows = slice(lo, min(n, lo + 2048))
            x, t = s[name][rows].double(), turn[rows]
            size = (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / D + EPS) ** 0.5
            y[rows] = _exact_turned(x / size * w, t, c["interleaved"])
            if dx is None:
                continue
            g = _exact_turned(s[d_out][rows].double(), t.conj(), c["interleaved"])
            dw += (g * x / size).flatten(0, 1).sum(0)
            gw = g * w
            dx[rows] = gw / size - x * (gw * x).sum(-1, keepdim=True) / (D * size ** 3)
        out[name] = y
        if dx is not None:
            out["d" + name], out["d" + name + "_weight"] = dx, dw
    if c["op"] == "norm_train":
        return {k: out[k] for k in ("q", "k", "dq", "dk", "dq_weight", "dk_weight")}
    answer = {"q": out["q"]}
    for name, rows, scale in (("k_pages", out["k"], s["k_scale"]), ("v_pages", s["v"].double(), s["v_scale"])):
        pool = torch.zeros(s[name].shape, dtype=torch.float64, device=DEVICE)
        x = rows[:n]
        if c["fp8"]:
            x = (x / scale.double()[:, None]).clamp(-448, 448)
        pool.view(-1, c["hkv"], D)[s["slot_map"][:n]] = x
        answer[name] = pool
    return {**answer, "k": out["k"]} if c["k_out"] else answer


def _exact_logprobs(c, s):
    rows, vocab, k = c["rows"], c["vocab"], c["top"]
    out = {name: torch.zeros(rows, dtype=torch.float64, device=DEVICE) for name in ("logprobs", "entropy", "lse")}
    if k:
        out.update(top_ids=None, top_logprobs=torch.full((rows, k), -math.inf, dtype=torch.float64, device=DEVICE))
    if c["op"] == "logprobs_train":
        out["d_logits"] = torch.zeros((rows, vocab), dtype=torch.float64, device=DEVICE)
    step = max(1, (1 << 26) // vocab)
    for lo in range(0, rows, step):
        part = slice(lo, min(rows, lo + step))
        has = s["tokens"][part] >= 0
        if not bool(has.any()):
            continue
        index = torch.arange(rows, device=DEVICE)[part][has]
        scale = s["row_scale"][index].double()[:, None] if c["scaled"] else 1.0
        z = s["logits"][index].double() * scale
        lse = torch.logsumexp(z, dim=-1)
        p = torch.softmax(z, dim=-1)
        token = s["tokens"][index]
        each = torch.arange(len(index), device=DEVICE)
        h = -torch.special.xlogy(p, p).sum(-1)
        out["lse"][index], out["entropy"][index] = lse, h
        out["logprobs"][index] = z[each, token] - lse
        if k:
            # (no order of equal logits matters here)
            best = z.topk(k, dim=-1).values
            out["top_logprobs"][index] = best - lse[:, None]
        if c["op"] == "logprobs_train":
            dg, dh = s["d_logprobs"][index].double(), s["d_entropy"][index].double()
            d = -dg[:, None] * p - dh[:, None] * (torch.special.xlogy(p, p) + p * h[:, None])
            d[each, token] += dg
            out["d_logits"][index] = d * scale
    return out
