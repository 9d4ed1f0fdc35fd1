"""Whole-prompt attention over scores of any size that float32 holds, on the GPU.

A query row has one dimension that is not zero, 1, so a score is its key's entry there, exactly. Among entries of 100 and
more, two that differ do so by at least 1/2 (bf16 has 8 bits), or by far more; what is left of a softmax is the mean over
the keys that share the largest one, with neighbours where they are close, and the tolerances are the ordinary ones of
``check_rows``: a probability of two neighbours of 100 is off by less than 2^-13 by the rounding of scale times maximum.
"""

import numpy as np
import pytest
import torch

from oracle import step
from paper_2609_08368_amd import rl_attn as ra
from tests.test_gpu_step import DEV, bits, check_rows, dev, rand

pytestmark = pytest.mark.gpu

SIZES = [1e2, 1e5, 3e7, 1e9, 5e9, 1e10, 1e12, 1e20, 1e30, 1e38]


def scores(rng, size, n, kind):
    x = rng.choice([-1.0, -0.5, 0.0, 0.5, 1.0], n) * size
    if kind == "rising":
        x = np.linspace(-1, 1, n) * size
    elif kind == "falling":
        x = np.linspace(1, -1, n) * size
    elif kind == "alike":
        x = np.full(n, size)
    elif kind == "low":
        x = np.full(n, -size)
    elif kind == "late":
        x = np.where(np.arange(n) > 70, size, 1.0)
    elif kind == "early":
        x = np.where(np.arange(n) < 3, size, 1.0)
    elif kind == "second":                                # keys 32 to 63 alone, the second half of a split step
        x = np.where((np.arange(n) // 32) == 1, -size, 1.0)
    return x


@pytest.mark.parametrize("hq,hkv", [(2, 1), (4, 1), (8, 2)], ids=["64", "128", "256"])   # rows a tile, with 256 CUs
def test_prefill_of_scores_of_any_size(hq, hkv):
    rng = np.random.default_rng(1)
    kinds = ["any", "rising", "falling", "alike", "low", "late", "early", "second"]
    cases = [scores(rng, size, 110, kind) for size in SIZES for kind in kinds]
    lens = [len(c) for c in cases]
    indptr = np.concatenate([[0], np.cumsum(lens)])
    rows = int(indptr[-1])
    q = torch.zeros((rows, hq, 128), dtype=torch.bfloat16, device=DEV)
    q[:, :, 100] = 1.0
    k = torch.zeros((rows, hkv, 128), dtype=torch.bfloat16, device=DEV)
    k[:, :, 100] = torch.from_numpy(np.concatenate(cases)).to(DEV, torch.bfloat16)[:, None]
    v = rand(6, rows, hkv, 128)
    for scale in (float(np.float32(np.log(2.0))), 0.75):
        ref = step.prefill(bits(q), bits(k), bits(v), indptr, scale)
        for dtype in (torch.bfloat16, torch.float32):
            out, lse = torch.empty(q.shape, dtype=dtype, device=DEV), torch.empty(q.shape[:2], device=DEV)
            ra.prefill(q, k, v, dev(indptr), scale, out=out, lse=lse)
            torch.cuda.synchronize()
            at = 0
            for i, n in enumerate(lens):
                part = slice(at, at + n)
                check_rows(out[part], lse[part], *(r[part] for r in ref), f32=dtype == torch.float32,
                           what=f"{SIZES[i // len(kinds)]:g} {kinds[i % len(kinds)]}, scale {scale}")
                at += n
    ra.check_device_errors()
