"""Entropies and log probabilities of rows with one sure token on the GPU (through the C-ABI): values near 0, held to what
sums in 32 bits next to 1 can give and no more.

A row has its largest logit m once, n others k below it and the rest so far below that their powers are zero; its scale is
ln 2 in fp32, so that the others' powers are 2^-k. With e = 2^-24 (half a step of fp32): the sum S of the powers, 2^y of y
around a base within 1/2 of the largest, is off relatively by 2 e of the largest's power and e of each of the n additions
that are not exact; its logarithm, at most 1/2, by e and the difference to the base by e; the mean of y by e / 2 for each
product and addition, n + 1 of them, and e of its quotient. Together at most (6 + 1.5 n) e; the others' powers are off by
(3 k + 20) e relatively, which the value itself, the sum of their parts, is as well.
"""

import numpy as np
import pytest
import torch

from oracle import ends
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_logprobs import DEV, E, KINDS, floats, tokens_of

pytestmark = pytest.mark.gpu

LARGEST = {"bf16": [30.25, -9.25, 0.75], "f32": [30.3125, -7.40625, 0.71875, 1000.59375, 5.0]}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("vocab", [64, 700, 5003, 20011, 100003])
def test_sure_rows(vocab, kind):
    H.say(f"sure rows {vocab} {kind}")
    rng = np.random.default_rng(vocab)
    cases = [(m, n, k) for m in LARGEST[kind] for n in (1, 3, 8) for k in (16, 18, 20, 22)]
    x = np.full((len(cases), vocab), -2.0 ** 15)
    tokens = np.zeros(len(cases), np.int64)
    for i, (m, n, k) in enumerate(cases):
        at = rng.permutation(vocab)[:n + 1]
        x[i, at], tokens[i] = m - k, at[0]
        x[i, at[0]] = m
    t = torch.from_numpy(x).to(DEV, KINDS[kind])
    assert np.array_equal(H.f64(t), x)                   # nothing is rounded on the way in
    scale = np.full(len(cases), np.log(2), np.float32)
    got, want = ra.token_logprobs(t, tokens_of(tokens), floats(scale), top=2), ends.token_logprobs(x, tokens, scale)
    ra.check_device_errors()
    n, k = (np.array([c[i] for c in cases]) for i in (1, 2))
    for name in ("entropy", "logprobs"):
        g, w = H.f64(getattr(got, name)), want[name]
        tol = E * (6 + 1.5 * n + (3 * k + 20) * np.abs(w))
        assert np.all(np.abs(g - w) <= tol), f"{name}: {np.max(np.abs(g - w) / tol)} of the bound"
    assert np.all(H.f64(got.entropy) >= 0) and np.array_equal(got.top_ids.cpu().numpy()[:, 0], tokens)
