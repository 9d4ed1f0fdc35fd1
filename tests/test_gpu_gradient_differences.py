"""Gradients against differences of the calls they belong to, along directions in which the gradients are large, with bounds
that wrong gradients (none, halved, negated, in another order, without a term of the formula) do not meet.

A difference F(x + d) - F(x - d) and the gradient along 2 d may differ by
* what the difference leaves out, which is computed: both in 64 bits, F's difference less the formula's gradient along 2 d;
* what the two calls of F are off by, and what the gradient is off by along 2 d, as counted where they are tested.
Nothing of this is taken from the results under test.
"""

import numpy as np
import pytest
import torch

from oracle import ends, step
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_logprobs import bounds, floats, tokens_of
from tests.test_gpu_logprobs_far import bound
from tests.test_gpu_norm_rope import normed_case, run_grad, weight
from tests.test_gpu_norm_rope import call as norm_rope
from tests.test_gpu_step import axes_of, dev, rand

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------------------------- log probabilities

def logits_case(seed, scale):
    """fp32 logits of which a few tokens have most of the probability, each row's token one of them."""
    rng = np.random.default_rng(seed)
    x = (rng.standard_normal((6, 333)) * 1.5).astype(np.float32)
    x[:, 40:43] += 4.0
    s = rng.uniform(0.5, 1.5, 6).astype(np.float32) if scale else None
    return x, rng.integers(40, 43, 6), s, rng.choice([-1.0, 1.0], 6), rng.choice([-0.7, 0.7], 6)


def value(f, g, h):
    lp, ent = (v if isinstance(v, np.ndarray) else H.f64(v) for v in (f["logprobs"], f["entropy"]))
    return g * lp + h * ent


@pytest.mark.parametrize("scale", [False, True])
@pytest.mark.parametrize("offset", [0.0, 2000.0])
@pytest.mark.parametrize("seed", range(3))
def test_gradient_of_log_probabilities(seed, offset, scale):
    x, tokens, s, g, h = logits_case(seed, scale)
    x = (x + np.float32(offset)).astype(np.float32)
    t, sd = tokens_of(tokens), floats(s)
    run = lambda y: ra.token_logprobs(floats(y), t, sd)._asdict()
    f = run(x)
    d = H.f64(ra.token_logprobs_backward(floats(x), t, f["lse"], floats(g), sd, entropy=f["entropy"], d_entropy=floats(h)))
    x64 = x.astype(np.float64)
    grad = ends.token_logprobs_backward(x64, tokens, g, h, s)
    off = bound(x64, tokens, g, h, s, "f32", grad, ends.token_logprobs(x64, tokens, s))
    wrong = {"none": 0 * grad, "half": grad / 2, "negated": -grad, "shifted": np.roll(grad, 1, axis=1),
             "of the entropy alone": ends.token_logprobs_backward(x64, tokens, 0 * g, h, s),
             "of the log probability alone": ends.token_logprobs_backward(x64, tokens, g, 0 * h, s)}
    met = {k: np.ones(6, bool) for k in wrong}
    rows, by = np.arange(6), np.float32(2.0 ** -4)
    for cols in (np.argsort(-x64, axis=1)[:, 0], np.argsort(-x64, axis=1)[:, 1], np.argsort(-x64, axis=1)[:, 2], tokens):
        up, down = x.copy(), x.copy()
        up[rows, cols] += by
        down[rows, cols] -= by
        moved = up.astype(np.float64)[rows, cols] - down.astype(np.float64)[rows, cols]
        exact = [value(ends.token_logprobs(y.astype(np.float64), tokens, s), g, h) for y in (up, down)]
        noise = 0
        for y in (up, down):
            tol_lp, _, tol_h = bounds(torch.from_numpy(y), tokens, s)
            noise = noise + np.abs(g) * tol_lp + np.abs(h) * tol_h
        tol = np.abs(exact[0] - exact[1] - grad[rows, cols] * moved) + noise + off[rows, cols] * moved
        diff = value(run(up), g, h) - value(run(down), g, h)
        assert np.all(np.abs(diff - d[rows, cols] * moved) <= tol)
        for k, w in wrong.items():
            met[k] &= np.abs(exact[0] - exact[1] - w[rows, cols] * moved) <= 2 * tol
    assert not any(m.any() for m in met.values()), met


# ------------------------------------------------------------------------------------------------ normed rotary rows

def along(a, b):
    return float((a * b).sum())


@pytest.mark.parametrize("name", ["q", "k"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_of_normed_rows(interleaved, name):
    """Rows and gradients of size 1. The outputs are rounded to half a step of bf16, 2^-8 of them, and off by 1e-5 before
    that; so is the gradient of the rows."""
    c = normed_case(8, 6, 4, 3, 64, axes_of("cycle", 64), f32=True)
    c["q"], c["k"] = rand(1, 6, 4, 128), rand(2, 6, 3, 128)
    i = "qk".index(name)
    dy = {"q": rand(3, 6, 4, 128), "k": rand(4, 6, 3, 128)}
    got = run_grad(c, dy["q"], dy["k"], interleaved=interleaved)
    got_dx, got_dw = H.f64(got[i]), H.f64(got[2 + i])
    x, w, y = H.f64(c[name]), weight(c, i), H.f64(dy[name])
    args = (c["eps"], c["pos"], c["freq"], c["axes"], interleaved)
    dx, dw = ends.norm_rope_backward(y, x, w, *args)
    n, r = ends._norm(x, float(np.float32(c["eps"])))
    turned_back = r * w * step.rope(y, *args[1:], inverse=True)                            # r u, no term of the mean
    mean = (turned_back * n).mean(axis=-1, keepdims=True)
    assert np.allclose(turned_back - n * mean, dx, rtol=0, atol=1e-9)
    rng = np.random.default_rng(5)
    shuffle = lambda v: rng.permutation(v.ravel()).reshape(v.shape)
    wrong = {"none": (0 * dx, 0 * dw), "half": (dx / 2, dw / 2), "twice": (2 * dx, 2 * dw), "negated": (-dx, -dw),
             "shuffled": (shuffle(dx), shuffle(dw)), "without the mean": (turned_back, None)}

    def check(move_x, move_w, name):
        """One direction; returns the wrong gradients that it tells."""
        ends_of = []
        for sign in (1, -1):
            cc = {**c, "w": list(c["w"])}
            cc[name] = (c[name].double() + sign * dev(move_x, torch.float64)).to(torch.bfloat16)
            cc["w"][i] = (c["w"][i].double() + sign * dev(move_w, torch.float64)).to(torch.float32)
            out = H.f64(norm_rope(cc, interleaved=interleaved)[i])
            exact = ends.norm_rope(H.f64(cc[name]), weight(cc, i), *args)
            ends_of.append((out, exact, H.f64(cc[name]), weight(cc, i)))
        (out0, exact0, x0, w0), (out1, exact1, x1, w1) = ends_of
        mx, mw = x0 - x1, w0 - w1
        truth = along(y, exact0 - exact1)
        noise = (2.0 ** -8 + 1e-5) * along(np.abs(y), np.abs(exact0) + np.abs(exact1))
        rounded = along((2.0 ** -8 + 1e-5) * np.abs(dx) + 1e-5 * np.abs(turned_back).mean(), np.abs(mx))
        rounded += 1e-5 * along(np.abs(y * n).sum(axis=(0, 1)) * 2, np.abs(mw))
        tol = abs(truth - along(dx, mx) - along(dw, mw)) + noise + rounded
        diff = along(y, out0 - out1)
        assert abs(diff - along(got_dx, mx) - along(got_dw, mw)) <= tol, (diff, tol)
        return {k for k, (a, b) in wrong.items() if abs(truth - along(a, mx) - along(dw if b is None else b, mw)) > 2 * tol}

    still = np.zeros(128)
    # along the gradient's signs; along each row, where only the mean's term keeps the gradient from changing; the weights'
    assert check(0.25 * np.sign(dx), still, name) >= {"none", "half", "twice", "negated", "shuffled"}
    assert check(0.25 * x * np.sign(mean), still, name) >= {"without the mean"}
    assert check(0 * x, 0.25 * np.sign(dw), name) >= {"none", "half", "twice", "negated", "shuffled"}
    ra.check_device_errors()
