"""Log probabilities of tokens, entropies, alternatives and the gradient of the logits on the GPU (through the C-ABI)
against their definition in 64 bits.

Tolerances, with e = 2^-24 (half a step of fp32). With y = (x - m) s log2 e, 2^y is off by 4 e |y ln 2| (difference,
constant, two products) and 2 e of the exponential; a sum over a row has at most 64 + 6 additions in a segment and a fold
of as many, each e of the sum of magnitudes. So with Y the mean of |y| under p, in nats:
  ln S by 200 e + 4 e Y; a log probability by that, the logarithm's 3 e (1 + ln S) and 4 e |x_token - m| s: together at
  most e (210 + 4 (Y + |z_token - m|) + 3 ln S);
  lse by that without the token and 2 e |lse|;
  the entropy by the error of ln S and of the mean of y, 2 (200 e + 4 e Y) Y: e (210 + 420 Y + 8 Y^2 + 3 ln S).
The gradient forms p from the rounded lse, so p is off relatively by dp = (the error of lse) + 2 e (|lse| + |ln p| + 2); its
terms by p (dp |g + h (ln p + H)| + |h| (dp + the error of H) + 4 e (|g| + |h| (|ln p| + H))), then half a step of the
output: 2^-8 of the value for bf16, 2^-24 for fp32 (a few for the products).
"""

import numpy as np
import pytest
import torch

from oracle import ends
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
KINDS = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(seed, rows, vocab, kind, sharp=3.0, pad=0, offset=0):
    """Rows of a buffer that is wider by `pad` columns and begins `offset` elements into its memory."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    flat = torch.empty(rows * (vocab + pad) + offset, dtype=KINDS[kind], device=DEV)
    x = flat[offset:].view(rows, vocab + pad)
    x.copy_(torch.randn(x.shape, generator=g, device=DEV) * sharp)
    rng = np.random.default_rng(seed)
    return x[:, :vocab], rng.integers(0, vocab, rows), rng


def tokens_of(t, kind=torch.int64):
    return torch.from_numpy(np.asarray(t)).to(DEV, kind)


def floats(x):
    return None if x is None else torch.from_numpy(np.asarray(x)).to(DEV, torch.float32)


def bounds(x, tokens, scale):
    """Of ln S, Y, |z_token - m| and lse (rows that have them)."""
    z = H.f64(x) * (1.0 if scale is None else np.asarray(scale, np.float32).astype(np.float64)[:, None])
    m = z.max(axis=-1, keepdims=True)
    w = np.exp(z - m)
    s = w.sum(axis=-1)
    y = np.where(w > 0, w * (m - np.maximum(z, -1e300)), 0).sum(axis=-1) / s
    at = np.abs(z[np.arange(len(z)), np.clip(tokens, 0, z.shape[1] - 1)] - m[:, 0])
    at = np.where(np.isfinite(at), at, 0)
    ln_s = np.log(s)
    tol_lp = E * (210 + 4 * (y + at) + 3 * ln_s)
    tol_lse = E * (210 + 4 * y + 3 * ln_s + 2 * np.abs(m[:, 0] + ln_s) + 2 * np.abs(m[:, 0]))
    tol_h = E * (210 + 420 * y + 8 * y * y + 3 * ln_s)
    # (rows without a token above -inf, or left out, answer with constants)
    return tuple(np.nan_to_num(t, nan=0.0) for t in (tol_lp, tol_lse, tol_h))


def check(got, x, tokens, scale=None, top=0):
    want = ends.token_logprobs(H.f64(x), tokens, scale, top)
    tol_lp, tol_lse, tol_h = bounds(x, tokens, scale)
    for name, tol in (("logprobs", tol_lp), ("lse", tol_lse), ("entropy", tol_h)):
        g, w = H.f64(getattr(got, name)), want[name]
        some = np.isfinite(w)
        assert np.array_equal(g[~some], w[~some], equal_nan=True), name
        assert np.all(np.abs(g - w)[some] <= tol[some]), f"{name}: {np.abs(g - w)[some]} of {tol[some]}"
        assert np.all(g[np.asarray(tokens) < 0] == 0)
    if top:
        assert np.array_equal(got.top_ids.cpu().numpy(), want["top_ids"])
        g, w = H.f64(got.top_logprobs), want["top_logprobs"]
        some = np.isfinite(w)
        tol = np.broadcast_to(tol_lse[:, None] + 4 * E * np.abs(np.where(some, w, 0)), w.shape)
        assert np.array_equal(g[~some], w[~some], equal_nan=True) and np.all(np.abs(g - w)[some] <= tol[some])
    if want["errors"]:
        with pytest.raises(ra.RlAttnError) as e:
            ra.check_device_errors()
        assert want["errors"] == set(str(e.value).split("):")[1].split()), str(e.value)
    else:
        ra.check_device_errors()
    return want


SHAPES = [(1, 1), (3, 2), (2, 7), (5, 63), (1, 64), (4, 257), (9, 1000), (3, 4095), (3, 4096), (3, 4097), (7, 16384),
          (2, 16385), (130, 5003), (1, 100003), (33, 40000), (1, 300007), (2500, 300)]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_matches_the_definition(shape, kind):
    rows, vocab = shape
    H.say(f"logprobs {shape} {kind}")
    x, tokens, rng = make(rows + vocab, rows, vocab, kind, pad=vocab % 3, offset=vocab % 5)
    check(ra.token_logprobs(x, tokens_of(tokens)), x, tokens)
    scale = rng.uniform(0.2, 3, rows).astype(np.float32)
    tokens[rows // 2] = -1
    for top in (1, 20, 32):
        check(ra.token_logprobs(x, tokens_of(tokens, torch.int32), floats(scale), top=top), x, tokens, scale, top)


@pytest.mark.parametrize("kind", list(KINDS))
def test_sharp_and_flat_rows(kind):
    """One sure token, ties everywhere, huge and tiny logits, equal rows of the type's lowest value."""
    vocab = 9001
    x, tokens, _ = make(1, 12, vocab, kind)
    x[0, 5000] = 60.0
    tokens[0] = 5000
    x[1] = 2.5
    x[2] = -0.0
    x[2, ::7] = 0.0
    x[3] = torch.finfo(x.dtype).min
    x[4] = torch.finfo(x.dtype).min
    x[4, 77:79] = 1.0
    tokens[4] = 78
    x[5] *= 1e30
    x[6] *= 1e-30
    x[7, :] = (torch.arange(vocab, device=DEV) // 40 % 7).to(x.dtype)   # 1300 largest logits
    x[8] = 1e4
    x[8, -1] = 10100.0
    for top in (0, 20, 32):
        check(ra.token_logprobs(x, tokens_of(tokens), top=top), x, tokens, None, top)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("vocab", [50, 9001, 40003])
def test_excluded_tokens_and_odd_values(vocab, kind):
    x, tokens, _ = make(2, 12, vocab, kind)
    inf = float("inf")
    x[0, ::2] = -inf
    tokens[0] = 2
    x[1] = -inf
    x[2] = -inf
    x[2, 41] = -3.0
    tokens[2] = 41
    x[3] = -inf
    x[3, 11:43] = 1.0
    x[4, 9] = float("nan")
    x[5, 9] = inf
    x[6, 3], x[6, 30] = inf, float("nan")
    x[7, 1:3] = inf
    x[8] = float("nan")
    x[9, : vocab - 1] = -inf
    x[10, 10:] = -inf
    x[10, :10] = float("nan")
    got = ra.token_logprobs(x, tokens_of(tokens), top=20)
    want = check(got, x, tokens, None, 20)
    assert np.isneginf(want["lse"][1]) and np.isnan(want["lse"][[4, 5, 6, 7, 8, 10]]).all()
    # only those rows
    fine, _, _ = make(2, 12, vocab, kind)
    assert torch.equal(ra.token_logprobs(fine, tokens_of(tokens)).logprobs[11], got.logprobs[11])


@pytest.mark.parametrize("kind", list(KINDS))
def test_tokens_and_scales_that_are_not_there(kind):
    x, tokens, rng = make(3, 9, 5000, kind)
    scale = rng.uniform(0.5, 2, 9).astype(np.float32)
    tokens[2], tokens[3], tokens[4] = 5000, -(1 << 40), 1 << 40
    check(ra.token_logprobs(x, tokens_of(tokens), floats(scale), top=3), x, tokens, scale, 3)
    tokens[2:5] = 1
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        scale[6] = bad
        check(ra.token_logprobs(x, tokens_of(tokens), floats(scale), top=3), x, tokens, scale, 3)
        d = ra.token_logprobs_backward(x, tokens_of(tokens), torch.zeros(9, device=DEV), torch.ones(9, device=DEV),
                                       floats(scale))
        assert torch.all(d[6] == 0) and torch.any(d[5] != 0)
        with pytest.raises(ra.RlAttnError, match="row-scale-invalid"):
            ra.check_device_errors()


@pytest.mark.parametrize("kind", list(KINDS))
def test_a_row_does_not_depend_on_its_call(kind):
    """Bits of a row among many and few others, at any place in memory, as a row of its own, beside asked alternatives."""
    vocab = 70001
    x, tokens, rng = make(4, 2100, vocab, kind)
    scale = rng.uniform(0.5, 2, 2100).astype(np.float32)
    t, s = tokens_of(tokens), floats(scale)
    many = ra.token_logprobs(x, t, s)
    for lo, n in ((0, 1), (5, 3), (100, 40), (1000, 700)):
        for top in (0, 20):
            few = ra.token_logprobs(x[lo:lo + n], t[lo:lo + n], s[lo:lo + n], top=top)
            for name in ("logprobs", "entropy", "lse"):
                assert torch.equal(getattr(few, name), getattr(many, name)[lo:lo + n]), (lo, n, name)
    for offset in (1, 3):
        moved = torch.empty(4 * vocab + offset, dtype=x.dtype, device=DEV)[offset:].view(4, vocab)
        moved.copy_(x[7:11])
        other = ra.token_logprobs(moved, t[7:11], s[7:11])
        assert torch.equal(other.logprobs, many.logprobs[7:11]) and torch.equal(other.entropy, many.entropy[7:11])


def test_broadcast_rows_and_strided_outputs():
    x, tokens, _ = make(5, 1, 3001, "f32")
    wide = x.expand(6, 3001)
    scale = floats([0.7]).expand(6)
    t = tokens_of(np.arange(6))
    got = ra.token_logprobs(wide, t, scale, top=4)
    want = ra.token_logprobs(wide.contiguous(), t, scale.contiguous(), top=4)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = torch.full((6, 3), -8.0, device=DEV)
    ids, lps = torch.full((6, 9), -8, dtype=torch.int32, device=DEV), torch.full((6, 9), -8.0, device=DEV)
    tt = torch.stack((t, t + 1), 1)[:, 0]
    ra.token_logprobs(wide, tt, scale, logprobs=out[:, 0], lse=out[:, 2], top_ids=ids[:, 2:6],
                      top_logprobs=lps[:, 3:7])
    assert torch.equal(out[:, 0], want.logprobs) and torch.equal(out[:, 2], want.lse) and torch.all(out[:, 1] == -8)
    assert torch.equal(ids[:, 2:6], want.top_ids) and torch.all(ids[:, :2] == -8) and torch.all(ids[:, 6:] == -8)
    assert torch.equal(lps[:, 3:7], want.top_logprobs)


def test_no_rows_and_every_row_left_out():
    x, _, _ = make(6, 5, 200, "bf16")
    got = ra.token_logprobs(x[:0], tokens_of(np.zeros(0, np.int64)), top=3)
    assert got.logprobs.shape == (0,) and got.top_ids.shape == (0, 3)
    got = ra.token_logprobs(x, tokens_of([-1] * 5), top=3)
    assert torch.all(got.lse == 0) and torch.all(got.top_ids == -1) and torch.all(got.top_logprobs == -float("inf"))


def test_alternatives_of_a_large_vocabulary():
    x, tokens, _ = make(7, 2, 1 << 21, "bf16")
    check(ra.token_logprobs(x, tokens_of(tokens), top=32), x, tokens, None, 32)


# ------------------------------------------------------------------------------------------------------- gradient

def check_grad(d, x, tokens, g, h, scale, kind, vocab):
    want = ends.token_logprobs_backward(H.f64(x), tokens, g, h, scale)
    f = ends.token_logprobs(H.f64(x), tokens, scale)
    _, tol_lse, tol_h = bounds(x, tokens, scale)
    s = 1.0 if scale is None else np.asarray(scale, np.float32).astype(np.float64)[:, None]
    with np.errstate(invalid="ignore"):
        lp = np.maximum(H.f64(x) * s - f["lse"][:, None], -1e4)
    p, hh = np.exp(lp), f["entropy"][:, None]
    ag, ah = np.abs(g)[:, None], np.abs(h)[:, None]
    dp = tol_lse[:, None] + 2 * E * (np.abs(f["lse"])[:, None] + np.abs(lp) + 2)
    tol = p * (dp * np.abs(g[:, None] + h[:, None] * (lp + hh)) + ah * (dp + tol_h[:, None])
               + 4 * E * (ag + ah * (np.abs(lp) + hh)))
    tol = s * tol + (2.0 ** -8 if kind == "bf16" else 4 * E) * np.abs(want) + 4 * E * s * (np.arange(vocab) == np.asarray(
        tokens)[:, None]) * ag + 1e-37
    got = H.f64(d)
    some = np.isfinite(f["lse"]) & (np.asarray(tokens) >= 0) & (np.asarray(tokens) < vocab)
    err = np.abs(got - want)[some]
    assert np.all(err <= tol[some]), f"{np.max(err / tol[some])} of the bound"
    assert np.all(got[np.isneginf(f["lse"]) | (np.asarray(tokens) < 0)] == 0)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (5, 63), (4, 257), (7, 4099), (3, 8192), (2, 16385), (70, 5003),
                                   (1, 100003)], ids=str)
def test_gradient_matches_the_formula(shape, kind):
    rows, vocab = shape
    H.say(f"logprobs gradient {shape} {kind}")
    x, tokens, rng = make(rows + vocab, rows, vocab, kind, pad=vocab % 3, offset=vocab % 5)
    scale = rng.uniform(0.3, 3, rows).astype(np.float32)
    g, h = rng.standard_normal(rows).astype(np.float32), rng.standard_normal(rows).astype(np.float32)
    if rows > 2:
        tokens[1] = -1
        x[2, vocab // 2:] = -float("inf")
    if rows > 4:
        x[3] = -float("inf")
        tokens[4] = min(3, vocab - 1)
    zero = np.zeros(rows)
    for sc, with_g, with_h in ((None, True, False), (scale, True, True), (scale, False, True)):
        f = ra.token_logprobs(x, tokens_of(tokens), floats(sc))
        d = ra.token_logprobs_backward(x, tokens_of(tokens), f.lse, floats(g) if with_g else None, floats(sc),
                                       entropy=f.entropy, d_entropy=floats(h) if with_h else None)
        check_grad(d, x, tokens, g.astype(np.float64) if with_g else zero, h.astype(np.float64) if with_h else zero, sc,
                   kind, vocab)
    # in place, and into a wider buffer whose other columns stay
    wide = torch.full((rows, vocab + 5), -8.0, dtype=x.dtype, device=DEV)
    args = (tokens_of(tokens), f.lse, None, floats(scale))
    ra.token_logprobs_backward(x, *args, entropy=f.entropy, d_entropy=floats(h), d_logits=wide[:, 2:vocab + 2])
    assert torch.equal(wide[:, 2:vocab + 2], d) and torch.all(wide[:, :2] == -8) and torch.all(wide[:, -3:] == -8)
    y = x.clone()
    assert ra.token_logprobs_backward(y, *args, entropy=f.entropy, d_entropy=floats(h), d_logits=y) is y
    assert torch.equal(y, d)
    ra.check_device_errors()


def test_gradient_of_broadcast_and_expanded_gradients():
    """One loss gradient for all rows, one row of logits for all tokens: gradients of the copies add up to the row's."""
    x, _, _ = make(9, 1, 501, "f32")
    tokens = np.arange(40) * 11 % 501
    wide = x.expand(40, 501)
    f = ra.token_logprobs(wide, tokens_of(tokens))
    one = torch.ones(1, device=DEV).expand(40)
    d = ra.token_logprobs_backward(wide, tokens_of(tokens), f.lse, one)
    p = torch.softmax(x[0].double(), 0)
    want = torch.zeros(501, dtype=torch.float64, device=DEV)
    want.scatter_add_(0, tokens_of(tokens), torch.ones(40, dtype=torch.float64, device=DEV))
    # 40 terms, each off by some 250 e of p and e of one
    assert torch.all((d.double().sum(0) - (want - 40 * p)).abs() <= 40 * (300 * E * p + 2 * E))


def test_gradient_is_the_difference_of_the_kernel():
    """Central differences of fp32 log probabilities: two errors of at most 300 e over a step of 2^-6, and the third
    derivative, 2^-12 / 6 of at most 1."""
    x, tokens, rng = make(10, 6, 333, "f32", sharp=1.5)
    g = rng.standard_normal(6).astype(np.float32)
    f = ra.token_logprobs(x, tokens_of(tokens))
    d = ra.token_logprobs_backward(x, tokens_of(tokens), f.lse, floats(g), entropy=f.entropy, d_entropy=floats(g))
    step = 2.0 ** -6
    for j in (0, 7, 332, int(tokens[0])):
        move = torch.zeros_like(x)
        move[:, j] = step
        a, b = (ra.token_logprobs(x + s * move, tokens_of(tokens)) for s in (1, -1))
        diff = ((a.logprobs - b.logprobs) + (a.entropy - b.entropy)).double() / (2 * step) * floats(g).double()
        bound = np.abs(g) * (2 * (300 + 420 * 6) * E / (2 * step) + 2.0 ** -12 * 8 / 6)
        assert np.all(np.abs(H.f64(d[:, j]) - H.f64(diff)) <= bound)


def test_outputs_that_are_not_asked_for():
    """The C call without entropy, lse or alternatives, and a gradient of the entropy alone."""
    import ctypes

    x, tokens, _ = make(11, 5, 20011, "bf16")
    t, want = tokens_of(tokens), ra.token_logprobs(x, tokens_of(tokens), top=2)
    lp = torch.empty(5, device=DEV)
    views = [None if v is None else ctypes.byref(ra.view(v)) for v in (x, t, None, lp, None, None, None, None)]
    assert ra.lib().rl_attn_token_logprobs(*views, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(lp, want.logprobs)


def test_the_same_call_gives_the_same_bits():
    """Rows that many workgroups share: whichever arrives last."""
    x, tokens, _ = make(12, 7, 250007, "bf16")
    t = tokens_of(tokens)
    first = ra.token_logprobs(x, t, top=32)
    for _ in range(200):
        assert all(torch.equal(a, b) for a, b in zip(ra.token_logprobs(x, t, top=32), first))


def test_logits_past_four_gigabytes():
    """Offsets beyond 32 bits in elements: the last rows give the bits that they give alone, forward and backward."""
    rows, vocab = 17001, 131073                          # 2.2e9 logits
    x = torch.zeros((rows, vocab), dtype=torch.bfloat16, device=DEV)
    some, tokens, _ = make(13, 3, vocab, "bf16")
    x[-3:] = some
    t = torch.full((rows,), 5, dtype=torch.int64, device=DEV)
    t[-3:] = tokens_of(tokens)
    got, alone = ra.token_logprobs(x, t), ra.token_logprobs(some, t[-3:])
    for name in ("logprobs", "entropy", "lse"):
        assert torch.equal(getattr(got, name)[-3:], getattr(alone, name))
    assert torch.all((got.lse[:-3] - np.log(vocab)).abs() < 1e-5)
    g = torch.ones(1, device=DEV).expand(rows)
    d = ra.token_logprobs_backward(some, t[-3:], alone.lse, g[:3])
    ra.token_logprobs_backward(x, t, got.lse, g, d_logits=x)
    assert torch.equal(x[-3:], d) and float(x[0, 5]) == pytest.approx(1.0, abs=2 ** -8)
    assert torch.all(x[rows - 4, 6:] == x[0, 6])        # (the last row of zeros)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("shape", [(3, 200), (3, 70001), (2050, 9001)], ids=str)
def test_signaling_nan_hides_no_alternative(shape, kind):
    """Every NaN pattern, in front of, behind and among a row's largest logits."""
    rows, vocab = shape
    x, tokens, _ = make(14, rows, vocab, kind)
    x[0, 64:72] = torch.arange(30, 38, device=DEV).to(x.dtype)
    x[1, :8] = 40.0
    bits = x.view(torch.int16 if kind == "bf16" else torch.int32)
    patterns = [0x7F81, 0x7FBF, -0x007F] if kind == "bf16" else [0x7F800001, 0x7FBFFFFF, -0x007FFFFF]
    for i, at in enumerate((63, 67, 68, 71, 72, 131, vocab - 1)):
        bits[0, at] = patterns[i % 3]
    bits[1, 4] = patterns[0]
    got = ra.token_logprobs(x, tokens_of(tokens), top=9)
    want = ends.token_logprobs(H.f64(x[:3]), tokens[:3], None, 9)
    assert np.array_equal(got.top_ids[:3].cpu().numpy(), want["top_ids"])
    assert torch.isnan(got.logprobs[:2]).all() and torch.isfinite(got.logprobs[2:]).all()
    ra.check_device_errors()


@pytest.mark.parametrize("vocab", [9001, 270001])
def test_alternatives_of_many_rows(vocab):
    """A workgroup to a row, of few and of many segments, gives what the workgroups that share a row give."""
    x, tokens, _ = make(15, 2100, vocab, "bf16")
    t = tokens_of(tokens)
    many = ra.token_logprobs(x, t, top=20)
    for lo in (0, 1000, 2093):
        few = ra.token_logprobs(x[lo:lo + 7], t[lo:lo + 7], top=20)
        assert torch.equal(few.top_ids, many.top_ids[lo:lo + 7])
        assert torch.equal(few.top_logprobs, many.top_logprobs[lo:lo + 7])
    check(few, x[2093:], tokens[2093:], None, 20)
