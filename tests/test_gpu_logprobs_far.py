"""The gradient of the logits for rows that lie far from zero or are scaled by a lot, on the GPU (through the C-ABI) against
its definition in 64 bits.

Tolerances, with e = 2^-24 (half a step of fp32), z = s x, m the largest z, Y the mean of |z - m| under p, H the entropy, S the
sum of exp(z - m). ln p_j is (x_j - m / s) s less ln S, or s x_j less an lse of magnitude up to 64, whose rounding is half a
step of [32, 64), 32 e. ln S is off by e (210 + 4 Y + 3 ln S), the terms by 2 e |z_j - m| (difference, product) and
e |ln p_j| (sum), the exponential by e |ln p_j| for each of the constant and the product and 2 e of its own:
  dp = e (246 + 4 Y + 3 ln S + 4 (|z_j - m| + |ln p_j|)) relative to p_j, without a term for the size of lse.
H is off by dh = e (210 + 420 Y + 8 Y^2 + 3 ln S). With a = |g + h (ln p + H)|, each of the three terms below rounded by
2 e: s p (dp a + |h| (dp + dh) + 4 e (|g| + |h| (|ln p| + H))), 4 e s |g| at the token, and half a step of the output:
2^-8 of the value for bf16, 4 e (with the products') for fp32.
"""

import numpy as np
import pytest
import torch

from oracle import ends
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_logprobs import DEV, E, KINDS, floats, make, tokens_of

pytestmark = pytest.mark.gpu


def bound(x, tokens, g, h, scale, kind, want, f):
    """Of each element of the gradient; f: what the forward call's definition gives."""
    s = (np.ones(len(x)) if scale is None else np.asarray(scale, np.float32).astype(np.float64))[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        z = x * s
        far = np.minimum(z.max(axis=-1, keepdims=True) - z, 1e4)
    w = np.exp(-far)
    total = w.sum(axis=-1, keepdims=True)
    y, ln_s, p = (w * far).sum(axis=-1, keepdims=True) / total, np.log(total), w / total
    lp, ent = np.abs(far + ln_s), f["entropy"][:, None]
    g, h = g[:, None], h[:, None]
    dp = E * (246 + 4 * y + 3 * ln_s + 4 * (far + lp))
    dh = E * (210 + 420 * y + 8 * y * y + 3 * ln_s)
    tol = p * (dp * np.abs(g + h * (ent - lp)) + np.abs(h) * (dp + dh) + 4 * E * (np.abs(g) + np.abs(h) * (lp + ent)))
    own = np.arange(x.shape[1]) == np.asarray(tokens)[:, None]
    # a power below 2^-126, the least normal number, may be taken as zero: p is off by that, and the output by as much
    tol = tol + 2.0 ** -126 * (np.abs(g) + np.abs(h) * (lp + ent))
    return s * (tol + 4 * E * np.abs(g) * own) + (2.0 ** -8 if kind == "bf16" else 4 * E) * np.abs(want) + 2.0 ** -126


def check(x, tokens, scale, g, h, kind, d):
    x64, g, h = H.f64(x), g.astype(np.float64), h.astype(np.float64)
    want = ends.token_logprobs_backward(x64, tokens, g, h, scale)
    f = ends.token_logprobs(x64, tokens, scale)
    tol, got = bound(x64, tokens, g, h, scale, kind, want, f), H.f64(d)
    some = np.isfinite(f["lse"]) & (np.asarray(tokens) >= 0)
    err = np.abs(got - want)
    worst = np.max((err / tol)[some], axis=-1)
    assert np.all(err[some] <= tol[some]), f"{worst} of the bound, lse {f['lse'][some]}"
    assert np.all(got[np.asarray(tokens) < 0] == 0)
    return f


def run(x, tokens, scale, g, h, **kw):
    t, s = tokens_of(tokens), floats(scale)
    f = ra.token_logprobs(x, t, s)
    d = ra.token_logprobs_backward(x, t, f.lse, floats(g), s, entropy=f.entropy, d_entropy=floats(h), **kw)
    ra.check_device_errors()
    return d


# (offset of the logits, scale): what a lse of 81, 700, 1e3, 7e3, 7e5, 7e8 and 1e7 does, logits of size 12 at scales of
# 1e2, 1e4 and 1e6, and the borders of the two ways that p is formed
PLACES = [(100, 0.7), (1000, 0.7), (1000, None), (-1000, 0.7), (1e4, 0.7), (1e6, 0.7), (1e9, None), (1e9, 0.7),
          (-1e9, 0.01), (0, 100.0), (0, 1e4), (0, 1e6), (0, None), (48, None), (-79, None), (1e-30, 1e30), (1e30, 1e-30)]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("place", PLACES, ids=str)
@pytest.mark.parametrize("shape", [(9, 5003), (3, 1), (2, 100003), (5, 63)], ids=str)
def test_gradient_at_any_offset_and_scale(shape, place, kind):
    rows, vocab = shape
    offset, scale = place
    H.say(f"logprobs gradient {shape} at {place} {kind}")
    x, tokens, rng = make(rows + vocab, rows, vocab, kind, sharp=4.0, pad=vocab % 3, offset=vocab % 5)
    if abs(offset) > 1e6:
        x *= abs(offset) * 2.0 ** -24                    # (so that the logits of a row differ in fp32)
    x += offset
    tokens[0] = int(H.f64(x[0]).argmax())
    if rows > 2:
        tokens[1] = -1
        x[2, 1 + vocab // 2:] = -float("inf")
    if rows > 4:
        x[3, tokens[3]] = -float("inf")
        x[4] = x[4, 0].clone()                           # all equal
    scale = None if scale is None else np.full(rows, scale, np.float32)
    g, h = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    d = run(x, tokens, scale, g, h)
    check(x, tokens, scale, g, h, kind, d)
    # in place, and into a wider buffer whose other columns stay
    wide = torch.full((rows, vocab + 5), -8.0, dtype=x.dtype, device=DEV)
    run(x, tokens, scale, g, h, d_logits=wide[:, 2:vocab + 2])
    assert torch.equal(wide[:, 2:vocab + 2], d) and torch.all(wide[:, :2] == -8) and torch.all(wide[:, -3:] == -8)
    y = x.clone()
    run(y, tokens, scale, g, h, d_logits=y)
    assert torch.equal(y, d)


@pytest.mark.parametrize("kind", list(KINDS))
def test_near_and_far_rows_of_one_call(kind):
    """Each row has the bits that it has alone, whatever the others are."""
    rows, vocab = 48, 20011
    x, tokens, rng = make(3, rows, vocab, kind)
    places = [0.0, 52.0, 1e3, -75.0, 80.0, -1e3, 5e4, 0.0]
    x += torch.tensor([places[i % 8] for i in range(rows)], device=DEV)[:, None].to(x.dtype)
    tokens[5::7] = -1
    x[11] = -float("inf")
    x[17, 4] = float("nan")
    scale = rng.uniform(0.5, 1.5, rows).astype(np.float32)
    g, h = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    d = run(x, tokens, scale, g, h)
    assert torch.isnan(d[17]).all() and torch.all(d[11] == 0)
    some = np.arange(rows) != 17
    f = check(x[some], tokens[some], scale[some], g[some], h[some], kind, d[torch.from_numpy(some).to(DEV)])
    assert np.abs(f["lse"][np.isfinite(f["lse"])]).max() > 1e3
    for lo, n in ((0, 1), (2, 1), (5, 4), (16, 2), (20, 28)):
        few = run(x[lo:lo + n], tokens[lo:lo + n], scale[lo:lo + n], g[lo:lo + n], h[lo:lo + n])
        assert torch.equal(few.view(torch.int16), d[lo:lo + n].view(torch.int16)), (lo, n)


def test_two_equal_logits_share_their_probability():
    x = torch.zeros((4, 700), device=DEV)
    for i, top in enumerate((1e3, 1e6, 1e9, -1e9)):
        x[i] = -3e38
        x[i, [3, 698]] = top
    one = torch.ones(4, device=DEV)
    t = tokens_of([3, 698, 3, 3])
    f = ra.token_logprobs(x, t)
    d = ra.token_logprobs_backward(x, t, f.lse, one)
    want = torch.zeros((4, 700), device=DEV)
    want[:, [3, 698]] = torch.tensor([0.5, -0.5], device=DEV)
    want[1] *= -1
    assert torch.all((d - want).abs() <= 4 * E)          # (two terms: nothing is rounded but a logarithm and its power)


def test_gradient_of_many_far_rows_and_of_a_large_vocabulary():
    for rows, vocab in ((2100, 301), (2, 1 << 21)):
        x, tokens, rng = make(rows, rows, vocab, "bf16")
        x += 5000
        g, h = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
        check(x, tokens, None, g, h, "bf16", run(x, tokens, None, g, h))


def test_gradient_of_far_rows_captured_and_replayed():
    x, tokens, _ = make(8, 40, 9001, "f32")
    x[::2] += 1e5
    t, one = tokens_of(tokens), torch.ones(40, device=DEV)
    f = ra.token_logprobs(x, t)
    want = ra.token_logprobs_backward(x, t, f.lse, one)
    d, s, graph = torch.zeros_like(x), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        ra.token_logprobs_backward(x, t, f.lse, one, d_logits=d)         # the stream's error word
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            ra.token_logprobs_backward(x, t, f.lse, one, d_logits=d)
        for _ in range(3):
            d.zero_()
            graph.replay()
            s.synchronize()
            assert torch.equal(d, want)


@pytest.mark.parametrize("kind", list(KINDS))
def test_gradient_of_rows_with_nan_anywhere(kind):
    """NaN at one place, in whole stretches of the row, beside excluded tokens: the whole row, whatever its other logits are."""
    x, tokens, rng = make(21, 12, 30011, kind)
    x[::2] += 1e4
    nan, inf = float("nan"), float("inf")
    for i, part in enumerate((slice(7, 8), slice(0, 8192), slice(4096, 20000), slice(30010, None), slice(None))):
        x[2 * i, part] = nan
        x[2 * i + 1, part] = nan
    x[4, 20000:] = -inf
    x[5, :4096] = -inf
    x[10, 3] = x[11, 3] = inf
    d = run(x, tokens, None, np.ones(12), np.ones(12))
    assert torch.isnan(d).all(dim=1).tolist() == [True] * 12
