"""The operators at a step's ends, written out plainly in 64 bits (test infrastructure).

* ``norm_rope`` -- a head's row over its root mean square, times the weights, then turned by its position; and its
  gradient ``norm_rope_backward``, from the chain rule.
* ``token_logprobs`` -- log softmax of given tokens, the entropy and the largest logits in order; and the gradient of the
  logits ``token_logprobs_backward``.
* ``fork_requests``, ``copy_pages``, ``drop_tokens`` -- a table of pages when requests begin as copies of others, and
  when they end: one request after the other, one page after the other.
"""

from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64
from .step import rope


def _norm(x, eps):
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return x * r, r


def norm_rope(x, weight, eps, positions, inv_freq, axes=None, interleaved=False):
    """``x`` ``[T, H, D]`` (bf16 bits or floats), ``weight`` ``[D]``; float64 ``[T, H, D]``."""
    n, _ = _norm(np.asarray(bf16_bits_to_f64(x), np.float64), float(np.float32(eps)))
    return rope(n * np.asarray(weight, np.float64), positions, inv_freq, axes, interleaved)


def norm_rope_backward(dy, x, weight, eps, positions, inv_freq, axes=None, interleaved=False):
    """``(dx, dweight)`` of ``norm_rope`` for the outputs' gradient ``dy``."""
    n, r = _norm(np.asarray(bf16_bits_to_f64(x), np.float64), float(np.float32(eps)))
    g = rope(dy, positions, inv_freq, axes, interleaved, inverse=True)
    u = g * np.asarray(weight, np.float64)
    return r * (u - n * (u * n).mean(axis=-1, keepdims=True)), (g * n).sum(axis=(0, 1))


def token_logprobs(logits, tokens, row_scale=None, top=0):
    """``logits`` ``[T, V]`` floats. A dict of ``logprobs``, ``entropy``, ``lse``, ``top_ids``, ``top_logprobs`` and
    ``errors``."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    out = {"logprobs": np.zeros(rows), "entropy": np.zeros(rows), "lse": np.zeros(rows),
           "top_ids": np.full((rows, top), -1), "top_logprobs": np.full((rows, top), -np.inf), "errors": set()}
    for t in range(rows):
        token, scale = int(tokens[t]), 1.0 if row_scale is None else float(np.float32(row_scale[t]))
        if token < 0:
            continue
        if token >= vocab:
            out["errors"].add("token-out-of-range")
        if not (scale > 0 and np.isfinite(scale)):
            out["errors"].add("row-scale-invalid")
        if token >= vocab or not (scale > 0 and np.isfinite(scale)):
            continue
        z = x[t] * scale
        if np.isnan(z).any() or np.isposinf(z).any():
            lse, lp, h = np.nan, np.full(vocab, np.nan), np.nan
        elif np.isneginf(z).all():
            lse, lp, h = -np.inf, z, 0.0
        else:
            # (around the maximum: the logits may be of any size)
            m = z.max()
            log_s = np.log(np.exp(z - m).sum())
            lse, lp = m + log_s, z - m - log_s
            p = np.exp(lp)
            h = -np.sum(p[p > 0] * lp[p > 0])
        out["lse"][t], out["logprobs"][t], out["entropy"][t] = lse, lp[token], h
        some = np.flatnonzero(x[t] > -np.inf)              # (not NaN either)
        best = some[np.argsort(-x[t, some], kind="stable")][:top]
        out["top_ids"][t, :len(best)] = best
        out["top_logprobs"][t, :len(best)] = lp[best]
    return out


def token_logprobs_backward(logits, tokens, d_logprobs, d_entropy, row_scale=None):
    """The gradient of ``sum(d_logprobs logprobs + d_entropy entropy)``."""
    x = np.asarray(logits, np.float64)
    f = token_logprobs(x, tokens, row_scale)
    d = np.zeros_like(x)
    for t in range(x.shape[0]):
        token, scale = int(tokens[t]), 1.0 if row_scale is None else float(np.float32(row_scale[t]))
        if token < 0 or token >= x.shape[1] or not (scale > 0 and np.isfinite(scale)) or np.isneginf(f["lse"][t]):
            continue
        with np.errstate(invalid="ignore"):
            z = x[t] * scale
            lp = z - z.max()
            lp = lp - np.log(np.exp(lp).sum())
            p = np.exp(lp)
            d[t] = -p * (d_logprobs[t] + d_entropy[t] * (np.maximum(lp, -1e4) + f["entropy"][t]))
        d[t, token] += d_logprobs[t]
        d[t] *= scale
    return d


def fork_requests(parents, fork_lens, kv_lens, free_pages, free_used, block_table, page_size, num_pages):
    """A dict of ``block_table``, ``kv_lens``, ``free_used``, ``copies`` (new arrays) and ``errors``."""
    table, lens = np.array(block_table, copy=True), np.array(kv_lens, np.int64)
    copies, errors = np.tile([-1, -1, 0], (len(lens), 1)), set()
    used, room = int(free_used), table.shape[1] * page_size
    if not 0 <= used <= len(free_pages):
        errors.add("free-pages-exhausted")
        used = min(max(used, 0), len(free_pages))
    over = False
    for b, p in enumerate(int(x) for x in parents):
        if p < 0:
            continue
        if p >= len(lens) or p == b or kv_lens[b] != 0 or parents[p] >= 0:
            errors.add("fork-invalid")
            continue
        n = int(fork_lens[b])
        if n < 0 or n > kv_lens[p] or kv_lens[p] > room:
            errors.add("length-out-of-range")
            continue
        full, rest = divmod(n, page_size)
        if rest and used == len(free_pages):
            over = True
        if over:
            errors.add("free-pages-exhausted")
            continue
        if rest:
            page = int(free_pages[used])
            used += 1
            if not 0 <= page < num_pages:
                errors.add("page-id-out-of-range")
                continue
            copies[b] = block_table[p, full], page, rest
            table[b, full] = page
        table[b, :full] = block_table[p, :full]
        lens[b] = n
    return {"block_table": table, "kv_lens": lens, "free_used": used, "copies": copies, "errors": errors}


def copy_pages(copies, pages):
    """The pool (any element type) after the copies."""
    out = np.array(pages, copy=True)
    for src, dst, rows in copies:
        if rows > 0:
            out[dst, :rows] = pages[src, :rows]
    return out


def drop_tokens(kv_lens, keep_lens, block_table, free_pages, free_used, page_size, num_pages):
    """A dict of ``free_pages``, ``kv_lens``, ``free_used`` (new arrays) and ``errors``."""
    kept, dropped, errors = set(), set(), set()
    out, lens = np.array(free_pages, copy=True), np.array(kv_lens, np.int64)
    room, used = block_table.shape[1] * page_size, int(free_used)
    if not 0 <= used <= len(free_pages):
        errors.add("free-pages-exhausted")
        used = min(max(used, 0), len(free_pages))
    for b, (kv, keep) in enumerate(zip(kv_lens, keep_lens)):
        if kv < 0 or kv > room or keep < 0:
            errors.add("length-out-of-range")
        have = min(max(int(kv), 0), room)
        stay = have if keep < 0 else min(int(keep), have)
        lens[b] = kv if keep < 0 else min(kv, keep)
        for j in range(-(-have // page_size)):
            page = int(block_table[b, j])
            if not 0 <= page < num_pages:
                errors.add("page-id-out-of-range")
            else:
                (kept if j < -(-stay // page_size) else dropped).add(page)
    freed = sorted(dropped - kept)
    if len(freed) > used:
        errors.add("free-pages-exhausted")
        freed = freed[len(freed) - used:]
    out[used - len(freed):used] = freed
    return {"free_pages": out, "kv_lens": lens, "free_used": used - len(freed), "errors": errors}
