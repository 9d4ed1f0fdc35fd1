"""Whole-prompt attention whose largest scores come late, in either half of a step's keys, on the GPU.

The prefill kernel takes a row's probabilities against the maximum of the row's first keys, and where a tile is split
between two waves (tiles of 64 and 128 rows) each wave against that of its own first keys: of 0-31 and of 32-63. Here the
two are up to 260 powers of two apart and later keys bring the lower half back to the upper one's weight.

Scores are exact but for the scale: a query row has one dimension that is not zero, a power of two, and a key's entry in
it is the score in powers of two (a whole number below 2^8, exact in bf16). The scale is the float32 next to ln 2; times
log2 e, both rounded to 32 bits and so is their product, an exponent is off by less than 2^-23 of itself, and its
difference to the first keys' maximum rounds by 2^-16 once more: below 2^-14 powers of two together, which moves a
probability by less than the 2^-12 that the tolerances of ``check_rows`` leave for the scores.
"""

import numpy as np
import pytest
import torch

from oracle import step
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_step import DEV, bits, check_rows, dev, rand

pytestmark = pytest.mark.gpu

SCALE = float(np.float32(np.log(2.0)))
GAPS = [0, 40, 90, 100, 119, 120, 121, 124, 125, 126, 127, 128, 129, 140, 180, 221, 223, 250]


def scores(gap, late_in, first_of_low):
    """A prompt's scores: the first keys of one half of a step at 0, of the other at ``gap``; from key 64 on, the lower
    half (``late_in`` keys behind) rises to the gap's height."""
    n = 64 + 64 + 17
    t = np.arange(n)
    low = (t % 64 < 32) if first_of_low == 0 else (t % 64 >= 32)
    s = np.where(low, 0.0, -20.0)
    s[63 if first_of_low == 0 else 5] = gap            # one key of the upper half's first ones
    # (weights 2^-3 each, a few keys of the lower half, so that the two halves weigh about the same)
    rise = low & (t >= 64 + late_in)
    s[np.flatnonzero(rise)[:6]] = gap - 3 if gap > 3 else gap
    return s


@pytest.mark.parametrize("hq,hkv", [(2, 1), (4, 1), (8, 2)], ids=["64", "128", "256"])   # rows a tile, with 256 CUs
def test_prefill_joins_halves_that_are_far_apart(hq, hkv):
    cases = [scores(g, late, f) for g in GAPS for late in (0, 33) for f in (0, 1)]
    lens = [len(c) for c in cases]
    indptr = np.concatenate([[0], np.cumsum(lens)])
    rows = int(indptr[-1])
    q = torch.zeros((rows, hq, 128), dtype=torch.bfloat16, device=DEV)
    q[:, :, 7] = torch.tensor([1.0, 0.5], device=DEV).repeat_interleave((hq + 1) // 2)[:hq].to(torch.bfloat16)
    k = torch.zeros((rows, hkv, 128), dtype=torch.bfloat16, device=DEV)
    k[:, :, 7] = torch.from_numpy(np.concatenate(cases)).to(DEV, torch.bfloat16)[:, None]
    assert np.array_equal(H.f64(k[:, 0, 7]), np.concatenate(cases)), "the scores are what was asked for"
    v = rand(5, rows, hkv, 128)
    ref = step.prefill(bits(q), bits(k), bits(v), indptr, SCALE)
    for dtype in (torch.bfloat16, torch.float32):
        out, lse = torch.empty(q.shape, dtype=dtype, device=DEV), torch.empty(q.shape[:2], device=DEV)
        ra.prefill(q, k, v, dev(indptr), SCALE, out=out, lse=lse)
        torch.cuda.synchronize()
        at = 0
        for i, n in enumerate(lens):
            rows_of = slice(at, at + n)
            check_rows(out[rows_of], lse[rows_of], *(r[rows_of] for r in ref), f32=dtype == torch.float32,
                       what=f"gap {GAPS[i // 4]}, late {i // 2 % 2}, low half {i % 2}")
            at += n
    ra.check_device_errors()
