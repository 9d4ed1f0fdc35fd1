"""A step's slot maps, rotary positions and whole-prompt attention, written out plainly (test infrastructure).

* ``map_slots`` -- where the new rows of a step go (paper, section "Fast Agentic Rollout with SGLang": a turn appends
  its suffix to cached context): pages are taken from the list of free ones in request order, a request that is invalid
  gets nothing, and from the first that does not fit on none does.
* ``rope`` -- rotary position embedding (Su et al., 2021) with an axis for each frequency: each pair of dimensions is a
  complex number multiplied by ``exp(i position frequency)``.
* ``prefill`` -- causal attention over packed rows of whole prompts: the definition of ``extend`` from an empty cache,
  without pages.
"""

from __future__ import annotations

import numpy as np

from .attention import _masked_attend, bf16_bits_to_f64


def map_slots(kv_lens, new_lens, free_pages, free_used, block_table, page_size, num_pages, rows, pos_delta=None):
    """Returns a dict of ``block_table``, ``kv_lens``, ``free_used``, ``qo_indptr``, ``slot_map``, ``positions`` (new
    arrays) and ``errors``, the set of what was wrong."""
    table = np.array(block_table, copy=True)
    room = table.shape[1] * page_size
    lens = [int(x) for x in kv_lens]
    used, taken = int(free_used), 0
    slots, pos = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    indptr, errors = [0], set()
    if not 0 <= used <= len(free_pages):
        errors.add("free-pages-exhausted")
        used = min(max(used, 0), len(free_pages))
    stopped = False
    for b, (c, n) in enumerate(zip(list(lens), (int(x) for x in new_lens))):
        if c < 0 or n < 0 or c + n > room:
            errors.add("length-out-of-range")
            n = 0
            need = 0
        else:
            need = -(-(c + n) // page_size) - -(-c // page_size)
        if not stopped and (indptr[-1] + n > rows or taken + need > len(free_pages) - used):
            errors.add("rows-past-slot-map" if indptr[-1] + n > rows else "free-pages-exhausted")
            stopped = True
        if stopped:
            n = need = 0
        for i in range(n):
            t = c + i
            j = t // page_size
            if j >= -(-c // page_size):
                page = int(free_pages[used + taken + j - -(-c // page_size)])
                if 0 <= page < num_pages:
                    table[b, j] = page
            else:
                page = int(table[b, j])
            r = indptr[-1] + i
            pos[r] = t + (0 if pos_delta is None else int(pos_delta[b]))
            if 0 <= page < num_pages:
                slots[r] = page * page_size + t % page_size
            else:
                errors.add("page-id-out-of-range")
        taken += need
        lens[b] = c + n
        indptr.append(indptr[-1] + n)
    return {"block_table": table, "kv_lens": np.array(lens, np.int64), "free_used": used + taken,
            "qo_indptr": np.array(indptr, np.int64), "slot_map": slots, "positions": pos, "errors": errors}


def rope(x, positions, inv_freq, axes=None, interleaved=False, inverse=False):
    """``x`` ``[T, H, D]`` (bf16 bits or floats) turned by ``positions`` ``[A, T]``; float64 ``[T, H, D]``."""
    y = np.array(bf16_bits_to_f64(x), dtype=np.float64)
    f = np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    n = len(f)
    which = np.zeros(n, np.int64) if axes is None else np.asarray(axes, dtype=np.int64)
    angle = np.asarray(positions, dtype=np.float64)[which].T * f
    turn = np.exp((-1j if inverse else 1j) * angle)[:, None, :]
    i = np.arange(n)
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
    z = (y[..., lo] + 1j * y[..., hi]) * turn
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def prefill(q, k, v, seq_indptr, scale, row_block: int = 64):
    """q ``[T, Hq, D]``, k, v ``[T, Hkv, D]`` (bf16 bits or floats). Returns ``(out, lse, spread)`` in float64, zero in
    rows that no prompt owns; ``spread`` is the same average of the values' magnitudes, which bounds what rounding the
    probabilities can do."""
    qf, kf, vf = (bf16_bits_to_f64(x) for x in (q, k, v))
    total, hq, d = qf.shape
    r = hq // kf.shape[1]
    out, spread, lse = np.zeros((total, hq, d)), np.zeros((total, hq, d)), np.zeros((total, hq))
    for q0, q1 in zip(seq_indptr[:-1], seq_indptr[1:]):
        for g in range(kf.shape[1]):
            heads = slice(g * r, (g + 1) * r)
            for i0 in range(int(q0), int(q1), row_block):
                i1 = min(int(q1), i0 + row_block)
                rows = qf[i0:i1, heads].reshape(-1, d)
                limits = np.repeat(np.arange(i0, i1) - int(q0), r)
                kk, vv = kf[q0:i1, g], vf[q0:i1, g]
                o, l = _masked_attend(rows, kk, vv, scale, limits)
                a, _ = _masked_attend(rows, kk, np.abs(vv), scale, limits)
                out[i0:i1, heads], spread[i0:i1, heads] = o.reshape(-1, r, d), a.reshape(-1, r, d)
                lse[i0:i1, heads] = l.reshape(-1, r)
    return out, lse, spread
