"""Normed rotary rows, alone, with their append and their gradient, on the GPU (through the C-ABI) against their
definition in 64 bits.

Tolerances, with e = 2^-24 (half a step of fp32). The sum of 128 squares is formed over at most 19 additions and
products, so it is off by 20 e relatively, its root by 10 e, the hardware's 1 / sqrt by 2 e more: r is off by 12 e, n =
r x by 13 e, w n by 14 e: less than 1e-6 of it. A rotated element is off by 5e-7 (|x| + |y|) of its pair beside
(tests/test_gpu_step.py), so by 1.5e-6 (|x| + |y|) in all, and by half a step more: 2^-8 of it for bf16.

Gradient: g, the output's gradient turned back, is off by dg = 5e-7 (|x| + |y|) of its pair; u = w g by w dg and e; the
mean of u n by the mean of w dg |n| and of (13 + 20 + 2) e |u n|; d_x = r (u - n mean) by r (w dg + |n| mean(w dg |n|)
+ 5e-6 (|u| + |n| mean |u n|)) at most, as 12 + 13 + 35 + 4 = 64 steps e are 4e-6; and half a step of bf16. A weight's
gradient sums g n over all rows: its terms are off by |n| dg + 14 e |g n|, and a sum of L terms one after the other in
each lane, then of trees of 6 + 2 + 3 levels around 128 terms one after the other, by (L + 140) e of the sum of
magnitudes.
"""

import numpy as np
import pytest
import torch

import oracle
from oracle import ends, step
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_step import AXES, append_case, axes_of, bits, dev, magnitude, rand, rope_args, rope_case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def normed_case(seed, rows, hq, hkv, freqs, axes, f32=False, far=0):
    c = rope_case(seed, rows, hq, hkv, freqs, axes, far)
    rng = np.random.default_rng(seed)
    for n in "qk":
        c[n] = (c[n].float() * dev(rng.uniform(0.01, 30, c[n].shape[1]), torch.float32)[:, None]).to(torch.bfloat16)
    kind = torch.float32 if f32 else torch.bfloat16
    c["w"] = [dev(rng.uniform(-0.5, 2.0, 128), kind) for _ in range(2)]
    c["eps"] = EPS
    return c


def weight(c, i):
    return c["w"][i].double().cpu().numpy()


def reference(c, name, interleaved):
    """(the rows, |x| + |y| of the normed pairs, |normed row|)"""
    i = "qk".index(name)
    x = H.f64(c[name])
    ref = ends.norm_rope(x, weight(c, i), c["eps"], c["pos"], c["freq"], c["axes"], interleaved)
    n = ends._norm(x, float(np.float32(c["eps"])))[0] * weight(c, i)
    return ref, np.maximum(magnitude(n, len(c["freq"]), interleaved), np.abs(n))


def check_normed(got, c, name, interleaved, rows=slice(None)):
    ref, mag = reference(c, name, interleaved)
    # (half a step of bf16's subnormals, which are multiples of 2^-133, is 2^-134)
    tol = 2.0 ** -8 * (np.abs(ref) + 1.5e-6 * mag) + 1.5e-6 * mag + 2.0 ** -134
    err = np.abs(H.f64(got) - ref)
    assert np.all(err[rows] <= tol[rows]), f"{name}: off by {np.max((err - tol)[rows])}"


def call(c, k=True, **kw):
    (pos, freq), axes = rope_args(c)
    return ra.norm_rope(c["q"], c["k"] if k else None, c["w"][0], c["w"][1] if k else None, c["eps"], pos, freq, axes,
                        **kw)


SIZES = [(1, 1, 1, 64), (3, 8, 2, 32), (5, 96, 8, 8), (130, 12, 1, 48), (67, 16, 16, 56), (700, 17, 3, 64)]


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_norm_rope_matches_the_definition(size, f32):
    rows, hq, hkv, freqs = size
    for interleaved in (False, True):
        kind = list(AXES)[(rows + interleaved) % 3]
        H.say(f"norm rope {size} {kind} interleaved={interleaved}")
        c = normed_case(rows + hq, rows, hq, hkv, freqs, axes_of(kind, freqs), f32, far=rows * 1000)
        q, k = call(c, interleaved=interleaved)
        check_normed(q, c, "q", interleaved)
        check_normed(k, c, "k", interleaved)
        q1, none = call(c, k=False, interleaved=interleaved)
        assert none is None and torch.equal(q1, q)
        # in place, in a fused buffer whose values stay
        fused = torch.cat((c["q"], c["k"], c["v"]), dim=1)
        d = {**c, "q": fused[:, :hq], "k": fused[:, hq:hq + hkv]}
        call(d, interleaved=interleaved, q_out=d["q"], k_out=d["k"])
        assert torch.equal(fused, torch.cat((q, k, c["v"]), dim=1))
    ra.check_device_errors()


def test_rows_of_any_size():
    """Zero rows, tiny and huge elements, an eps above the row, NaN and infinities: of their own row alone."""
    c = normed_case(3, 12, 2, 1, 64, None)
    q = c["q"]
    q[0], q[1], q[2], q[3] = 0, 1e-30, 1e18, torch.tensor(3e-39).to(torch.bfloat16)
    check_normed(call(c)[0], c, "q", False)
    check_normed(call({**c, "eps": 100.0})[0], {**c, "eps": 100.0}, "q", False)
    plain = call(c)[0]
    q[5, 0, 17], q[6, 1, 3], q[7, 0, 100] = float("nan"), float("inf"), -float("inf")
    got = call(c)[0]
    assert torch.isnan(got[5, 0]).all() and not torch.isfinite(got[6, 1]).all()
    odd = torch.zeros(12, 2, dtype=torch.bool, device=DEV)
    odd[5, 0] = odd[6, 1] = odd[7, 0] = True
    assert torch.equal(got[~odd], plain[~odd])


def test_a_row_does_not_depend_on_its_call():
    """Calls of few and of many rows run differently shared out."""
    c = normed_case(5, 3000, 64, 8, 64, axes_of("cycle", 64))
    (pos, freq), axes = rope_args(c)
    q, k = call(c)
    for lo, n in ((0, 1), (17, 100), (2400, 600)):
        few = ra.norm_rope(c["q"][lo:lo + n], c["k"][lo:lo + n], *c["w"], EPS, pos[:, lo:lo + n], freq, axes)
        assert torch.equal(few[0], q[lo:lo + n]) and torch.equal(few[1], k[lo:lo + n])


def run_append(c, interleaved, q_out, k_out, pools):
    (pos, freq), axes = rope_args(c)
    f = ra.norm_rope_append_kv_fp8 if c["scales"] else ra.norm_rope_append_kv
    return f(c["q"], c["k"], c["v"], *c["w"], EPS, pos, freq, dev(c["slots"], torch.int64), *pools, *c["scales"], axes,
             interleaved=interleaved, q_out=q_out, k_out=k_out)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("size", [(1, 8, 2, 64, 8, 0), (6, 96, 8, 64, 64, 3), (130, 12, 1, 32, 16, 1),
                                  (77, 16, 16, 40, 128, 60), (901, 64, 8, 64, 64, 11)], ids=str)
def test_append_writes_rows_and_pages(size, fp8):
    rows, hq, hkv, freqs, page, pad = size
    interleaved, kind = rows % 2 == 0, ("text", "blocks", "cycle")[rows % 3]
    H.say(f"norm rope append {size} fp8={fp8}")
    c = append_case(rows, rows, hq, hkv, freqs, axes_of(kind, freqs), page, fp8, pad)
    c.update(w=normed_case(rows, 1, 1, 1, 8, None, f32=rows % 3 == 1)["w"], eps=EPS)
    pools = [p.clone() for p in c["pools"]]
    marks = [torch.full_like(c[n], 7.0) for n in "qk"]
    q, k = (m.clone() for m in marks)
    run_append(c, interleaved, q, k, pools)
    ra.check_device_errors()
    real, tail = slice(0, rows), slice(rows, None)
    check_normed(q, c, "q", interleaved, real)
    check_normed(k, c, "k", interleaved, real)
    alone = call(c, interleaved=interleaved)
    assert torch.equal(q[real], alone[0][real]) and torch.equal(k[real], alone[1][real])
    assert torch.equal(q[tail], marks[0][tail]) and torch.equal(k[tail], marks[1][tail])
    slots = torch.from_numpy(c["slots"][real]).to(DEV)
    flat = [p.view(torch.uint8).view(-1, hkv, 128 * (1 if fp8 else 2)) for p in pools]
    rest = torch.ones(flat[0].shape[0], dtype=torch.bool, device=DEV)
    rest[slots] = False
    for p, before in zip(flat, c["pools"]):
        assert torch.equal(p[rest], before.view(torch.uint8).view(p.shape)[rest])
    if not fp8:
        assert torch.equal(flat[0][slots], k[real].view(torch.uint8))
        assert torch.equal(flat[1][slots], c["v"][real].contiguous().view(torch.uint8))
    else:
        want = oracle.quantize_rows(bits(c["v"][real].contiguous()), c["scales"][1].cpu().numpy())
        assert np.array_equal(flat[1][slots].cpu().numpy(), want)
        ref, mag = (x[real] for x in reference(c, "k", interleaved))
        s = c["scales"][0].cpu().numpy().astype(np.float64)[:, None]
        ref = np.clip(ref / s, -448, 448)
        got = oracle.fp8_e4m3_to_f64(flat[0][slots].cpu().numpy())
        slack = 1.5e-6 * mag / s + 2.0 ** -23 * np.abs(ref)      # the element's and the quotient's own error
        assert np.all(np.abs(got - ref) <= np.maximum(2.0 ** -4 * (np.abs(ref) + slack), 2.0 ** -10) + slack)
    again = [p.clone() for p in c["pools"]]
    q2 = c["q"].clone()
    run_append({**c, "q": q2}, interleaved, q2, None, again)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(again, pools))
    assert torch.equal(q2[real], q[real]) and torch.equal(q2[tail], c["q"][tail])


# ------------------------------------------------------------------------------------------------------- gradient

def run_grad(c, dq_out, dk_out, k=True, **kw):
    (pos, freq), axes = rope_args(c)
    return ra.norm_rope_backward(dq_out, dk_out if k else None, c["q"], c["k"] if k else None, c["w"][0],
                                 c["w"][1] if k else None, c["eps"], pos, freq, axes, **kw)


def check_grad(got_dx, got_dw, dy, c, name, interleaved):
    i = "qk".index(name)
    x, w, y = H.f64(c[name]), weight(c, i), H.f64(dy)
    dx, dw = ends.norm_rope_backward(y, x, w, c["eps"], c["pos"], c["freq"], c["axes"], interleaved)
    n, r = ends._norm(x, float(np.float32(c["eps"])))
    dg = 5e-7 * magnitude(y, len(c["freq"]), interleaved)
    g = step.rope(y, c["pos"], c["freq"], c["axes"], interleaved, inverse=True)
    u, a = np.abs(w * g), np.abs(n)
    mean = lambda v: v.mean(axis=-1, keepdims=True)
    tol = r * (np.abs(w) * dg + a * mean(np.abs(w) * dg * a) + 5e-6 * (u + a * mean(u * a)))
    tol = tol + 2.0 ** -8 * (np.abs(dx) + tol)
    err = np.abs(H.f64(got_dx) - dx)
    assert np.all(err <= tol), f"d{name}: off by {np.max(err - tol)}"
    if got_dw is None:
        return
    lane = -(-x.shape[0] * -(-x.shape[1] // 8) // 4) // max(1, min(900, x.shape[0] * x.shape[1] // 32)) + 1
    size = np.abs(g * n).sum(axis=(0, 1))
    tol = (a * dg).sum(axis=(0, 1)) + (14 + lane + 140) * 2.0 ** -24 * size
    err = np.abs(H.f64(got_dw) - dw)
    assert np.all(err <= tol), f"d{name}_weight: off by {np.max(err - tol)}"


@pytest.mark.parametrize("f32", [False, True], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES + [(2111, 32, 8, 64)], ids=str)
def test_gradient_matches_the_formula(size, f32):
    rows, hq, hkv, freqs = size
    interleaved, kind = (rows + hq + f32) % 2 == 0, list(AXES)[(rows + f32) % 3]
    H.say(f"norm rope gradient {size} {kind} interleaved={interleaved}")
    c = normed_case(rows + hq, rows, hq, hkv, freqs, axes_of(kind, freqs), f32, far=rows * 1000)
    dq_out, dk_out = rand(rows + 7, rows, hq, 128), rand(rows + 8, rows, hkv, 128)
    got = run_grad(c, dq_out, dk_out, interleaved=interleaved)
    check_grad(got.dq, got.dq_weight, dq_out, c, "q", interleaved)
    check_grad(got.dk, got.dk_weight, dk_out, c, "k", interleaved)
    again = run_grad(c, dq_out, dk_out, interleaved=interleaved)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    # without k; in place
    alone = run_grad(c, dq_out, None, k=False, interleaved=interleaved)
    assert alone.dk is None and alone.dk_weight is None and torch.equal(alone.dq, got.dq)
    check_grad(alone.dq, alone.dq_weight, dq_out, c, "q", interleaved)
    g = torch.cat((dq_out, dk_out), dim=1)
    run_grad(c, g[:, :hq], g[:, hq:], interleaved=interleaved, dq=g[:, :hq], dk=g[:, hq:])
    assert torch.equal(g, torch.cat((got.dq, got.dk), dim=1))
    ra.check_device_errors()


def test_gradient_of_the_kernel_is_its_difference():
    """Along a direction that moves elements by whole steps of bf16; the outputs' steps of 2^-8 of some 2000 elements add
    up like a random walk: sum d_out out moves by less than 6 sigma of 2^-8 |d_out out| / sqrt(3) a side."""
    c = normed_case(8, 4, 4, 2, 64, None)
    c["q"], c["k"] = rand(1, 4, 4, 128), rand(2, 4, 2, 128)
    dq_out = rand(3, 4, 4, 128)
    d = (rand(4, 4, 4, 128).float() * 0.25).to(torch.bfloat16)
    out = [call({**c, "q": c["q"] + s * d}, k=False)[0].double() for s in (1, -1)]
    moved = ((c["q"] + d).double() - (c["q"] - d).double())
    noise = 2.0 ** -8 / 3 ** 0.5 * torch.sqrt(((dq_out.double() * out[0]) ** 2).sum() * 2)
    got = run_grad(c, dq_out, None, k=False)
    along = (got.dq.double() * moved).sum()
    want = (dq_out.double() * (out[0] - out[1])).sum()
    # and the step's third derivative: (step / row's size)^2, at most 0.25^2, of the sum of magnitudes
    curve = 0.25 ** 2 * (got.dq.double() * moved).abs().sum()
    assert abs(along - want) <= 6 * noise + curve, (float(along), float(want), float(noise), float(curve))


def test_gradient_of_expanded_and_strange_rows():
    """One gradient row for all heads, rows in another order in memory, no rows at all."""
    c = normed_case(9, 40, 8, 2, 64, axes_of("blocks", 64))
    one = rand(1, 40, 1, 128)
    wide = one.expand(40, 8, 128)
    got = run_grad(c, wide, rand(2, 40, 2, 128))
    want = run_grad(c, wide.contiguous(), rand(2, 40, 2, 128))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    turned = {**c, "q": c["q"].transpose(0, 1).contiguous().transpose(0, 1)}
    dq = torch.empty(8, 40, 128, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    other = run_grad(turned, wide, rand(2, 40, 2, 128), dq=dq)
    assert all(torch.equal(x, y) for x, y in zip(other, got))
    none = {**c, "q": c["q"][:0], "k": c["k"][:0], "pos": c["pos"][:, :0]}
    got = run_grad(none, wide[:0], rand(2, 40, 2, 128)[:0])
    assert torch.equal(got.dq_weight, torch.zeros(128, device=DEV)) and torch.all(got.dk_weight == 0)
    few = {**c, "q": c["q"][:, :0]}
    got = run_grad(few, wide[:, :0], rand(2, 40, 2, 128))
    assert torch.all(got.dq_weight == 0) and torch.equal(got.dk, want.dk)


def test_gradient_reports_an_axis_that_is_not_there():
    c = normed_case(7, 5, 2, 2, 16, axes_of("cycle", 16))
    bad = {**c, "axes": np.where(np.arange(16) == 2, 7, c["axes"])}
    got = run_grad(bad, rand(1, 5, 2, 128), rand(2, 5, 2, 128))
    want = run_grad({**c, "axes": np.clip(bad["axes"], 0, 2)}, rand(1, 5, 2, 128), rand(2, 5, 2, 128))
    assert torch.equal(got.dq, want.dq)
    with pytest.raises(ra.RlAttnError) as e:
        ra.check_device_errors()
    assert "position-axis-out-of-range" in str(e.value)
