"""A step's slot maps, rotary rows and whole-prompt attention on the GPU (through the C-ABI) against their definitions
in 64 bits.

Tolerances. Slot maps are whole numbers and equal. A rotated element is formed in fp32 from a cosine and a sine off by
less than 2e-7 (the angle's rounding 5e-8, the polynomial and its evaluation below 1.5e-7) with two products and a sum
(half a step of 6e-8 each), so it is off by at most 5e-7 (|x| + |y|) before it is rounded, and by half a step more
after: 2^-8 of the value for bf16; for E4M3 2^-4 of the quotient, or 2^-10 (half the subnormal step). Attention rounds
the probabilities to bf16 (2^-8 of each, so 2^-8 of the average of the values' magnitudes), the result to bf16 (2^-8 of
it), and a score by the fp32 sum of 128 products: at most 128 * 2^-24 * sum |q k| scale, which is below 2^-13 for these
inputs and moves a probability by twice that relatively.
"""

import numpy as np
import pytest
import torch

from oracle import step
from paper_2609_08368_amd import rl_attn as ra
from paper_2609_08368_amd import workloads as wl
from tests import gpu_helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(x, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV, dtype)


def rand(seed, *shape, spread=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * spread).to(torch.bfloat16)


def bits(t):
    return wl.to_numpy_bits(t)


# ------------------------------------------------------------------------------------------------------ slot maps

def map_case(seed, batch, cached_hi, new_hi, page, pad=0, new_lo=0, used=5):
    rng = np.random.default_rng(seed)
    cached, new = rng.integers(0, cached_hi + 1, batch), rng.integers(new_lo, new_hi + 1, batch)
    before, after = -(-cached // page), -(-(cached + new) // page)
    pool = int(after.sum()) + 9
    ids = rng.permutation(pool)
    table = np.full((batch, int(after.max()) + 2 if batch else 2), -5)
    table[np.arange(table.shape[1])[None] < before[:, None]] = ids[:int(before.sum())]
    free = np.concatenate([rng.integers(0, pool, used), ids[int(before.sum()):]])
    return dict(kv_lens=cached, new_lens=new, free_pages=free, free_used=used, block_table=table, page_size=page,
                num_pages=pool, rows=int(new.sum()) + pad, pos_delta=rng.integers(-9, 9, batch))


def run_map(c, in_place=False, stream=None):
    t = {k: dev(c[k]) for k in ("kv_lens", "new_lens", "free_pages", "block_table")}
    used = dev(np.array([c["free_used"]]))
    delta = None if c["pos_delta"] is None else dev(c["pos_delta"])
    more = dict(kv_lens_out=t["kv_lens"], free_used_out=used) if in_place else {}
    m = ra.map_slots(t["kv_lens"], t["new_lens"], t["free_pages"], used, t["block_table"], c["page_size"],
                     c["num_pages"], slot_map=torch.full((c["rows"],), -99, dtype=torch.int64, device=DEV),
                     pos_delta=delta, **more)
    torch.cuda.synchronize()
    return {**{k: v.cpu().numpy() for k, v in m._asdict().items()}, "block_table": t["block_table"].cpu().numpy(),
            "before": t["kv_lens"].cpu().numpy()}


def check_map(c, in_place=False):
    want, got = step.map_slots(**c), run_map(c, in_place)
    for k in ("block_table", "kv_lens", "qo_indptr", "slot_map", "positions"):
        assert np.array_equal(got[k], want[k]), k
    assert int(got["free_used"][0]) == want["free_used"]
    if not in_place:
        assert np.array_equal(got["before"], c["kv_lens"]), "the lengths before the step are left as they were"
    if want["errors"]:
        with pytest.raises(ra.RlAttnError) as e:
            ra.check_device_errors()
        assert want["errors"] == set(str(e.value).split("):")[1].split()), str(e.value)
    else:
        ra.check_device_errors()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", [
    (1, 300, 1, 64), (1, 0, 1, 8), (1, 0, 1025, 128), (7, 500, 40, 16), (128, 4000, 1, 64), (32, 9000, 2048, 64),
    (1023, 60, 9, 8), (1024, 60, 1, 16), (1025, 60, 1, 16), (3001, 90, 3, 32), (2500, 700, 33, 8)], ids=str)
def test_map_equals_the_definition(case, in_place):
    batch, cached, new, page = case
    H.say(f"map {case} in_place={in_place}")
    for pad in (0, 37):
        check_map(map_case(sum(case) + pad, batch, cached, new, page, pad, new_lo=int(new == 1)), in_place)


def test_map_of_nothing():
    for c in (map_case(1, 0, 0, 0, 8, pad=3), map_case(2, 5, 50, 0, 8, pad=3), map_case(3, 5, 50, 0, 8)):
        check_map({**c, "pos_delta": None})


@pytest.mark.parametrize("change", [
    lambda c: c["kv_lens"].__setitem__(2, -1), lambda c: c["new_lens"].__setitem__(2, -3),
    lambda c: c["new_lens"].__setitem__(2, 10 ** 9), lambda c: c["kv_lens"].__setitem__(2, 2 ** 31 - 1),
    lambda c: c.update(rows=c["rows"] - 1), lambda c: c.update(rows=7), lambda c: c.update(rows=0),
    lambda c: c.update(free_pages=c["free_pages"][:-12]), lambda c: c.update(free_used=10 ** 6),
    lambda c: c.update(free_used=-4), lambda c: c.update(free_pages=c["free_pages"][:0], free_used=0),
    lambda c: c["free_pages"].__setitem__(9, -1), lambda c: c["free_pages"].__setitem__(9, 10 ** 9),
    lambda c: c["block_table"].__setitem__((slice(None), slice(0, 9)), -1)], ids=range(14))
@pytest.mark.parametrize("size", [(40, 100, 30, 16), (1500, 100, 5, 8)], ids=str)
def test_map_refuses_and_reports(change, size):
    c = map_case(11, *size)
    change(c)
    check_map(c, in_place=True)


def test_map_reads_strides():
    c = map_case(5, 20, 200, 50, 16, pad=3)
    want = step.map_slots(**c)
    wide = {k: dev(np.stack([c[k], c[k] * 0 - 8], 1)) for k in ("kv_lens", "new_lens", "free_pages", "pos_delta")}
    table = dev(np.full((c["block_table"].shape[1], 2, 20), -5))
    table[:, 1] = dev(c["block_table"]).T
    out = {k: torch.full((n, 3), -8, dtype=d, device=DEV) for k, n, d in (
        ("kv_lens_out", 20, torch.int32), ("qo_indptr", 21, torch.int32), ("slot_map", c["rows"], torch.int64),
        ("positions", c["rows"], torch.int32))}
    ra.map_slots(wide["kv_lens"][:, 0], wide["new_lens"][:, 0], wide["free_pages"][:, 0], dev(np.array([5])),
                 table[:, 1].T, 16, c["num_pages"], pos_delta=wide["pos_delta"][:, 0],
                 **{k: v[:, 1] for k, v in out.items()})
    for k, name in (("kv_lens_out", "kv_lens"), ("qo_indptr", "qo_indptr"), ("slot_map", "slot_map"),
                    ("positions", "positions")):
        assert np.array_equal(out[k][:, 1].cpu().numpy(), want[name]), k
        assert torch.all(out[k][:, ::2] == -8)
    assert np.array_equal(table[:, 1].T.cpu().numpy(), want["block_table"]) and torch.all(table[:, 0] == -5)


# ---------------------------------------------------------------------------------------------------- rotary rows

def rope_case(seed, rows, hq, hkv, freqs, axes, far=0):
    rng = np.random.default_rng(seed)
    n_axes = 1 if axes is None else int(np.max(axes)) + 1
    pos = rng.integers(-20, 3000, (n_axes, rows)) + far
    return dict(q=rand(seed, rows, hq, 128), k=rand(seed + 1, rows, hkv, 128), v=rand(seed + 2, rows, hkv, 128),
                pos=pos, freq=10000.0 ** (-np.arange(freqs) / freqs), axes=axes)


def magnitude(x, freqs, interleaved):
    """|x| + |y| of each element's pair (zero where nothing turns, so that the copy has to be exact)."""
    a = np.abs(x)
    m = np.zeros_like(a)
    i = np.arange(freqs)
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, freqs + i)
    m[..., lo] = m[..., hi] = a[..., lo] + a[..., hi]
    return m


def check_turned(got, x, c, interleaved, inverse=False, rows=slice(None), what=""):
    x = H.f64(x)
    freqs = len(c["freq"])
    ref = step.rope(x, c["pos"], c["freq"], c["axes"], interleaved, inverse)
    mag = magnitude(x, freqs, interleaved)
    tol = np.where(mag > 0, 2.0 ** -8 * (np.abs(ref) + 5e-7 * mag) + 5e-7 * mag, 0.0)
    err = np.abs(H.f64(got) - ref)
    assert np.all(err[rows] <= tol[rows]), f"{what}: off by {np.max((err - tol)[rows])}"


AXES = {"text": None, "blocks": lambda n: np.repeat([0, 1, 2], [n - 2 * (3 * n // 8), 3 * n // 8, 3 * n // 8]),
        "cycle": lambda n: np.arange(n) % 3}


def axes_of(kind, n):
    return None if AXES[kind] is None else AXES[kind](n)


def rope_args(c):
    return (dev(c["pos"]), dev(c["freq"], torch.float32)), None if c["axes"] is None else dev(c["axes"])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", list(AXES))
@pytest.mark.parametrize("size", [(1, 1, 1, 64), (3, 8, 2, 32), (5, 96, 8, 8), (130, 12, 1, 48), (67, 16, 16, 56)],
                         ids=str)
def test_rope_turns_rows(size, kind, interleaved):
    rows, hq, hkv, freqs = size
    H.say(f"rope {size} {kind} interleaved={interleaved}")
    c = rope_case(rows + hq, rows, hq, hkv, freqs, axes_of(kind, freqs))
    args, axes = rope_args(c)
    for inverse in (False, True):
        q, k = ra.rope(c["q"], c["k"], *args, axes, interleaved=interleaved, inverse=inverse)
        check_turned(q, c["q"], c, interleaved, inverse, what="q")
        check_turned(k, c["k"], c, interleaved, inverse, what="k")
    q1, none = ra.rope(c["q"], None, *args, axes, interleaved=interleaved, inverse=True)
    assert none is None and torch.equal(q1, q)
    # in place, in a fused buffer
    fused = torch.cat((c["q"], c["k"], c["v"]), dim=1)
    ra.rope(fused[:, :hq], fused[:, hq:hq + hkv], *args, axes, interleaved=interleaved, inverse=True,
            q_out=fused[:, :hq], k_out=fused[:, hq:hq + hkv])
    assert torch.equal(fused, torch.cat((q, k, c["v"]), dim=1))
    ra.check_device_errors()


@pytest.mark.parametrize("far", [65536, 1 << 20, 1 << 24, 2 ** 31 - 4000, -(2 ** 31) + 30])
def test_rope_of_far_positions(far):
    c = rope_case(3, 33, 4, 2, 64, axes_of("cycle", 64), far)
    args, axes = rope_args(c)
    q, k = ra.rope(c["q"], c["k"], *args, axes)
    check_turned(q, c["q"], c, False)
    check_turned(k, c["k"], c, False)


def test_rope_special_angles_and_values():
    """Quarter turns and their neighbours, zero and infinite frequencies, infinities and NaN in a row that turns."""
    freq = np.array([0.0, np.pi / 2, np.pi / 4, np.pi, 2 * np.pi, 1e-30, 3.0, -1.5], dtype=np.float32)
    c = dict(rope_case(4, 50, 2, 1, 8, None), freq=freq, pos=np.arange(-25, 25)[None])
    args, _ = rope_args(c)
    for interleaved in (False, True):
        q, _ = ra.rope(c["q"], None, *args, interleaved=interleaved)
        check_turned(q, c["q"], c, interleaved)
        assert torch.equal(q[25], c["q"][25]), "position zero turns nothing"
    x = c["q"].clone()
    x[3, 0, 100], x[4, 1, 101], x[5, 0, 2] = float("inf"), float("nan"), float("inf")
    q, _ = ra.rope(x, None, *args)
    assert torch.isinf(q[3, 0, 100]) and torch.isnan(q[4, 1, 101]) and not torch.isfinite(q[5, 0, 2])
    assert torch.isfinite(q).sum() == q.numel() - 4


def test_rope_reads_positions_of_any_stride():
    c = rope_case(6, 21, 4, 2, 16, axes_of("cycle", 16))
    args, axes = rope_args(c)
    one = args[0][:1]
    a = ra.rope(c["q"], c["k"], one.expand(3, -1), args[1], axes)
    b = ra.rope(c["q"], c["k"], one, args[1])
    turned = args[0].T.contiguous().T
    d, e = ra.rope(c["q"], c["k"], turned, args[1], axes), ra.rope(c["q"], c["k"], args[0], args[1], axes)
    for x, y in ((a, b), (d, e)):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_rope_reports_an_axis_that_is_not_there():
    c = rope_case(7, 5, 2, 2, 16, axes_of("cycle", 16))
    args, axes = rope_args(c)
    bad = axes.clone()
    bad[2], bad[4] = 7, -1
    q, _ = ra.rope(c["q"], c["k"], *args, bad)
    check_turned(q, c["q"], {**c, "axes": np.clip(bad.cpu().numpy(), 0, 2)}, False)
    with pytest.raises(ra.RlAttnError) as e:
        ra.check_device_errors()
    assert "position-axis-out-of-range" in str(e.value)


# ------------------------------------------------------------------------------------- rotary rows and their append

def append_case(seed, rows, hq, hkv, freqs, axes, page, fp8, pad):
    rng = np.random.default_rng(seed)
    c = rope_case(seed, rows + pad, hq, hkv, freqs, axes)
    pool = -(-(rows + page) // page) + 2
    order, at = rng.permutation(pool), np.arange(rows) + int(rng.integers(0, page))
    c["slots"] = np.concatenate([order[at // page] * page + at % page, np.full(pad, -1)])
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    c["pools"] = [rand(seed + i, pool, page, hkv, 128).to(kind) for i in (5, 6)]
    c["scales"] = [dev(rng.uniform(0.003, 0.03, hkv), torch.float32) for _ in range(2)] if fp8 else []
    return c


def run_append(c, interleaved, q_out, k_out, pools):
    (pos, freq), axes = rope_args(c)
    call = ra.rope_append_kv_fp8 if c["scales"] else ra.rope_append_kv
    return call(c["q"], c["k"], c["v"], pos, freq, dev(c["slots"], torch.int64), *pools, *c["scales"], axes,
                interleaved=interleaved, q_out=q_out, k_out=k_out)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("size", [(1, 8, 2, 64, 8, 0), (6, 96, 8, 64, 64, 3), (130, 12, 1, 32, 16, 1),
                                  (77, 16, 16, 40, 128, 60), (501, 64, 8, 64, 64, 11)], ids=str)
def test_rope_append_writes_rows_and_pages(size, fp8):
    rows, hq, hkv, freqs, page, pad = size
    interleaved, kind = rows % 2 == 0, ("text", "blocks", "cycle")[rows % 3]
    H.say(f"rope append {size} fp8={fp8}")
    c = append_case(rows, rows, hq, hkv, freqs, axes_of(kind, freqs), page, fp8, pad)
    pools = [p.clone() for p in c["pools"]]
    marks = [torch.full_like(c[n], 7.0) for n in "qk"]
    q, k = (m.clone() for m in marks)
    run_append(c, interleaved, q, k, pools)
    ra.check_device_errors()
    real, tail = slice(0, rows), slice(rows, None)
    check_turned(q, c["q"], c, interleaved, rows=real, what="q")
    check_turned(k, c["k"], c, interleaved, rows=real, what="k")
    assert torch.equal(q[tail], marks[0][tail]) and torch.equal(k[tail], marks[1][tail])
    # the rows of the pages, and nothing else of them
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
        import oracle

        want = oracle.quantize_rows(bits(c["v"][real].contiguous()), c["scales"][1].cpu().numpy())
        assert np.array_equal(flat[1][slots].cpu().numpy(), want)
        x = H.f64(c["k"])
        mag = magnitude(x, freqs, interleaved)[real]
        s = c["scales"][0].cpu().numpy().astype(np.float64)[:, None]
        ref = np.clip(step.rope(x, c["pos"], c["freq"], c["axes"], interleaved)[real] / s, -448, 448)
        got = oracle.fp8_e4m3_to_f64(flat[0][slots].cpu().numpy())
        slack = 5e-7 * mag / s + 2.0 ** -23 * np.abs(ref)        # the element's and the quotient's own error
        assert np.all(np.abs(got - ref) <= np.maximum(2.0 ** -4 * (np.abs(ref) + slack), 2.0 ** -10) + slack)
    # without rows of keys, and q in place: the same pages and rows
    again, held = [p.clone() for p in c["pools"]], c["q"]
    c["q"] = held.clone()
    run_append(c, interleaved, c["q"], None, again)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(again, pools))
    assert torch.equal(c["q"][real], q[real]) and torch.equal(c["q"][tail], held[tail])


@pytest.mark.parametrize("fp8", [False, True])
def test_rope_append_reports_slots_and_scales(fp8):
    c = append_case(9, 20, 4, 2, 64, None, 16, fp8, 0)
    limit = c["pools"][0].shape[0] * 16
    c["slots"][3], c["slots"][5], c["slots"][7] = limit, 1 << 40, -(1 << 40)
    pools, q = [p.clone() for p in c["pools"]], torch.full_like(c["q"], 7.0)
    run_append(c, False, q, None, pools)
    with pytest.raises(ra.RlAttnError) as e:
        ra.check_device_errors()
    assert "slot-out-of-range" in str(e.value)
    assert torch.all(q[7] == 7.0) and not torch.any(torch.all(q[[3, 5]] == 7.0, dim=-1))
    if fp8:
        c = append_case(10, 20, 4, 2, 64, None, 16, fp8, 0)
        for bad in (0.0, -1.0, float("nan"), float("inf")):
            c["scales"][0][1] = bad
            pools = [p.clone() for p in c["pools"]]
            run_append(c, False, None, None, pools)
            with pytest.raises(ra.RlAttnError) as e:
                ra.check_device_errors()
            assert "dequant-scale-invalid" in str(e.value)
            assert torch.equal(pools[0][:, :, 1].view(torch.uint8), c["pools"][0][:, :, 1].view(torch.uint8))


def test_rope_append_equals_rope_then_append():
    """bf16 pages: the pass writes what the two calls write."""
    c = append_case(12, 200, 16, 4, 64, axes_of("blocks", 64), 32, False, 0)
    (pos, freq), axes = rope_args(c)
    pools = [p.clone() for p in c["pools"]]
    q = run_append(c, False, None, None, pools)
    q2, k2 = ra.rope(c["q"], c["k"], pos, freq, axes)
    assert torch.equal(q, q2)
    flat = [p.clone().view(-1, 4, 128) for p in c["pools"]]
    flat[0][dev(c["slots"], torch.int64)], flat[1][dev(c["slots"], torch.int64)] = k2, c["v"]
    assert all(torch.equal(a.view(b.shape), b) for a, b in zip(pools, flat))


# ----------------------------------------------------------------------------------------------- whole prompts

def prompts(seed, lens, hq, hkv, pad=0, spread=None):
    indptr = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    rows = int(indptr[-1]) + pad
    q, k, v = rand(seed, rows, hq, 128), rand(seed + 1, rows, hkv, 128), rand(seed + 2, rows, hkv, 128)
    if spread is not None:
        k *= spread
    return dict(q=q, k=k, v=v, indptr=indptr, rows=rows)


def run_prefill(c, dtype=torch.bfloat16, lse=True, fill=float("nan")):
    out = torch.full(c["q"].shape, fill, dtype=dtype, device=DEV)
    l = torch.full(c["q"].shape[:2], fill, dtype=torch.float32, device=DEV) if lse else None
    ra.prefill(c["q"], c["k"], c["v"], dev(c["indptr"]), 128 ** -0.5, out=out, lse=l)
    torch.cuda.synchronize()
    return out, l


def check_rows(got, lse, ref, ref_lse, spread, f32=False, what=""):
    """Element by element, by the bound of the head of this file."""
    g = H.f64(got)
    assert np.all(np.isfinite(g)), f"{what}: not finite"
    tol = (2.0 ** -8 + 2.0 ** -12) * spread + (2.0 ** -22 if f32 else 2.0 ** -8) * np.abs(ref) + 1e-30
    off = np.abs(g - ref) / tol
    assert off.max(initial=0) <= 1.0, f"{what}: {off.max():.2f} of the bound"
    if lse is not None:
        d = np.abs(H.f64(lse) - ref_lse) / np.maximum(1.0, np.abs(ref_lse))
        assert d.max(initial=0) <= H.LSE_REL, f"{what}: lse off by {d.max():.2e}"


PROMPTS = [
    ([1], 1, 1), ([1], 8, 2), ([2, 1, 3], 8, 1), ([31, 32, 33], 8, 2), ([63, 64, 65, 1], 16, 2), ([0, 127, 0, 128, 129, 0], 8, 8),
    ([255, 256, 257], 4, 4), ([300, 5, 700], 12, 1), ([90] * 40, 16, 2), ([450], 96, 8), ([200, 333], 64, 2),
    ([513], 40, 2), ([77, 140], 20, 1), ([40], 256, 1), ([1025, 3], 24, 2), ([1] * 130 + [600], 8, 2)]


@pytest.mark.parametrize("case", PROMPTS, ids=[f"{len(c[0])}x{max(c[0])}_{c[1]}_{c[2]}" for c in PROMPTS])
def test_prefill_matches_the_definition(case):
    lens, hq, hkv = case
    H.say(f"prefill {lens[:8]} {hq}/{hkv}")
    c = prompts(sum(lens) + hq, lens, hq, hkv, pad=9)
    n = int(c["indptr"][-1])
    ref, ref_lse, spread = step.prefill(bits(c["q"]), bits(c["k"]), bits(c["v"]), c["indptr"], 128 ** -0.5)
    for dtype in (torch.bfloat16, torch.float32):
        out, lse = run_prefill(c, dtype)
        check_rows(out[:n], lse[:n], ref[:n], ref_lse[:n], spread[:n], dtype == torch.float32)
        assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all(), "rows of no prompt are left as they were"
    again, _ = run_prefill(c, torch.float32, lse=False)
    assert torch.equal(again[:n], out[:n])
    ra.check_device_errors()


def reference_rows(c, b, rows):
    """Rows of prompt b in 64 bits with torch on the GPU (too many for the plain loop): out, lse, spread."""
    q0 = int(c["indptr"][b])
    hq, hkv = c["q"].shape[1], c["k"].shape[1]
    outs = []
    for i in rows:
        k, v = (x[q0:q0 + i + 1].double().permute(1, 0, 2).contiguous() for x in (c["k"], c["v"]))
        q = c["q"][q0 + i].double().view(hkv, hq // hkv, 128)
        s = float(np.float32(128 ** -0.5)) * torch.matmul(q, k.transpose(1, 2).contiguous())
        lse = torch.logsumexp(s, dim=-1)
        p = torch.exp(s - lse[..., None])
        outs.append((torch.matmul(p, v).view(hq, 128), lse.view(hq), torch.matmul(p, v.abs()).view(hq, 128)))
    return tuple(np.stack([o[j].cpu().numpy() for o in outs]) for j in range(3))


@pytest.mark.parametrize("case", [([40000], 8, 1), ([20011, 3, 9000], 16, 2), ([6000] * 5, 64, 8)], ids=str)
def test_prefill_of_long_prompts(case):
    lens, hq, hkv = case
    H.say(f"prefill {case}")
    c = prompts(7, lens, hq, hkv)
    out, lse = run_prefill(c)
    assert torch.isfinite(out).all()
    for b, n in enumerate(lens):
        rows = sorted({0, n - 1, n // 2, *np.random.default_rng(b).integers(0, n, 12).tolist(),
                       *(r for r in (16383, 16384, 16385, 32767, 32768) if r < n)})
        ref = reference_rows(c, b, rows)
        at = torch.tensor([int(c["indptr"][b]) + r for r in rows], device=DEV)
        check_rows(out[at], lse[at], *ref, what=f"prompt {b}")


@pytest.mark.parametrize("hq,hkv", [(8, 2), (96, 8)])
def test_prefill_sees_nothing_behind_a_row(hq, hkv):
    """Infinities and NaN in a prompt's later rows, in other prompts and behind the last: earlier rows keep their bits."""
    lens = [150, 411, 60]
    c = prompts(21, lens, hq, hkv, pad=5)
    out, lse = run_prefill(c)
    for at, bad in ((400, float("nan")), (400, float("inf")), (151, float("nan")), (289, -float("inf")), (300, float("nan"))):
        for name in ("k", "v"):
            d = dict(c, **{name: c[name].clone()})
            d[name][at:at + 2] = bad
            d[name][int(c["indptr"][-1]):] = bad
            o, l = run_prefill(d)
            same = [r for r in range(int(c["indptr"][-1])) if r < at or r >= 561]
            ref = step.prefill(bits(c["q"]), bits(c["k"]), bits(c["v"]), c["indptr"], 128 ** -0.5)
            check_rows(o[same], l[same], ref[0][same], ref[1][same], ref[2][same], what=f"{name} {at} {bad}")
            if np.isnan(bad):
                assert torch.isnan(o[at]).all(), "and a row that sees it is not a number"


def test_prefill_of_extreme_scores():
    """Scores far apart (one key takes all), equal ones (the mean of the values), and far below zero."""
    c = prompts(31, [300], 8, 2)
    for factor in (0.0, 30.0, -200.0):
        d = dict(c, k=c["k"] * factor)
        if factor < 0:
            d["q"] = c["q"].abs()
            d["k"] = -c["k"].abs() * 50
        ref = step.prefill(bits(d["q"]), bits(d["k"]), bits(d["v"]), d["indptr"], 128 ** -0.5)
        out, lse = run_prefill(d)
        # (a score's own error grows with the sum of its products' magnitudes: 128 products, fp32)
        mag = np.abs(H.f64(d["q"])).sum(-1).max() * np.abs(H.f64(d["k"])).max() * 128 ** -0.5
        tol = (2.0 ** -8 + 2 * 128 * 2.0 ** -24 * mag) * ref[2] + 2.0 ** -8 * np.abs(ref[0])
        assert np.all(np.abs(H.f64(out) - ref[0]) <= tol), factor
        assert np.all(np.abs(H.f64(lse) - ref[1]) <= 1e-4 * np.maximum(1, np.abs(ref[1])))


# (prompts whose tiles have 64, 128 and 256 rows on a device of 256 CUs, and their neighbours in length)
@pytest.mark.parametrize("case", [
    ([511], 32, 8), ([513], 32, 8), ([2000], 32, 8), ([1500, 0, 500], 32, 8), ([2111], 32, 8), ([63, 65], 96, 96),
    ([129, 127], 64, 64), ([800], 128, 128), ([33, 1, 31], 5, 1), ([600], 128, 1), ([300, 40], 70, 1)], ids=str)
def test_prefill_of_every_tile(case):
    lens, hq, hkv = case
    c = prompts(sum(lens) + hq, lens, hq, hkv, pad=2)
    ref = step.prefill(bits(c["q"]), bits(c["k"]), bits(c["v"]), c["indptr"], 128 ** -0.5)
    rows = int(c["indptr"][-1])
    for dtype in (torch.bfloat16, torch.float32):
        out, lse = run_prefill(c, dtype)
        check_rows(out[:rows], lse[:rows], ref[0][:rows], ref[1][:rows], ref[2][:rows], f32=dtype == torch.float32,
                   what=f"{case}")
        assert torch.isnan(out[rows:].float()).all() and torch.isnan(lse[rows:]).all(), "rows behind the last prompt"
        again, _ = run_prefill(c, dtype)
        assert torch.equal(out[:rows], again[:rows]), "repeatable"


@pytest.mark.parametrize("hq,hkv", [(96, 96), (128, 64)])
def test_prefill_of_large_tiles_sees_nothing_behind_a_row(hq, hkv):
    test_prefill_sees_nothing_behind_a_row(hq, hkv)


@pytest.mark.parametrize("lens,hq,hkv", [([511], 32, 8), ([2000], 32, 8), ([800], 128, 128)], ids=str)
def test_prefill_of_scores_that_outgrow_the_first_keys(lens, hq, hkv):
    """A row's largest score comes late and lies hundreds above (or all lie far below) those of its first keys."""
    c = prompts(41, lens, hq, hkv)
    d = dict(c, q=c["q"].abs(), k=c["k"].abs().float())
    ramp = torch.linspace(-1.0, 1.0, lens[0], device=DEV)[:, None, None]
    for late in (ramp, -ramp, ramp.abs() - 0.5, torch.where(ramp > 0.5, 60.0, -60.0)):
        d["k"] = (c["k"].abs().float() * 40 * late).to(torch.bfloat16)
        ref = step.prefill(bits(d["q"]), bits(d["k"]), bits(d["v"]), d["indptr"], 128 ** -0.5)
        out, lse = run_prefill(d)
        mag = np.abs(H.f64(d["q"])).sum(-1).max() * np.abs(H.f64(d["k"])).max() * 128 ** -0.5
        tol = (2.0 ** -8 + 2 * 128 * 2.0 ** -24 * mag) * ref[2] + 2.0 ** -8 * np.abs(ref[0])
        assert np.all(np.abs(H.f64(out) - ref[0]) <= tol)
        assert np.all(np.abs(H.f64(lse) - ref[1]) <= 1e-4 * np.maximum(1, np.abs(ref[1])))


def test_prefill_reads_strides():
    c = prompts(41, [100, 37], 8, 2)
    want, want_lse = run_prefill(c)
    fused = torch.cat((c["q"], c["k"], c["v"]), dim=1)
    wide = torch.empty((c["rows"], 3, 20, 256), dtype=torch.bfloat16, device=DEV)
    wide[:, 1, 4:16, 64:192] = fused
    view = wide[:, 1, 4:16, 64:192]
    out = torch.zeros((8, c["rows"], 136), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((8, c["rows"] + 1), device=DEV)
    ptr = torch.stack((dev(c["indptr"]), dev(c["indptr"])), 1)[:, 0]
    ra.prefill(view[:, :8], view[:, 8:10], view[:, 10:], ptr, 128 ** -0.5, out=out[:, :, :128].transpose(0, 1),
               lse=lse[:, :-1].T)
    assert torch.equal(out[:, :, :128].transpose(0, 1), want) and torch.equal(lse[:, :-1].T, want_lse)
    assert torch.all(out[:, :, 128:] == 0) and torch.all(lse[:, -1] == 0)
    # one KV row and head for all: broadcast inputs
    one = c["k"][:1, :1].expand(c["rows"], 2, 128)
    o, _ = run_prefill(dict(c, k=one, v=c["v"]))
    o2, _ = run_prefill(dict(c, k=one.contiguous(), v=c["v"]))
    assert torch.equal(o, o2)


@pytest.mark.parametrize("indptr", [[0, 50, 40, 100], [-3, 20, 90], [0, 20, 140], [5, 20, 90], [0, 1 << 30], [90, 0]],
                         ids=str)
def test_prefill_clamps_and_reports_bounds(indptr):
    c = dict(prompts(51, [100], 8, 2), indptr=np.array(indptr))
    out, _ = run_prefill(c)
    bad = indptr[0] < 0 or indptr[-1] > 100 or any(b < a for a, b in zip(indptr, indptr[1:]))
    if bad:
        with pytest.raises(ra.RlAttnError) as e:
            ra.check_device_errors()
        assert "indptr-invalid" in str(e.value)
    else:
        ra.check_device_errors()
    if indptr == [5, 20, 90]:
        ref = step.prefill(bits(c["q"]), bits(c["k"]), bits(c["v"]), c["indptr"], 128 ** -0.5)
        assert torch.isnan(out[:5]).all() and torch.isnan(out[90:]).all()
        check_rows(out[5:90], None, ref[0][5:90], None, ref[2][5:90])


def test_prefill_agrees_with_extend():
    """The same rows in pages, extended from an empty cache."""
    lens = [333, 64, 1, 128]
    w = wl.custom(61, "extend", lens, q_lens=lens, hq=16, hkv=2, page_size=64)
    t = wl.materialize(w, DEV)
    o1, l1 = H.run_extend(w, t)
    k, v = (torch.cat([t[n][t["block_table"][b, :-(-m // 64)].long()].reshape(-1, 2, 128)[:m]
                       for b, m in enumerate(lens)]) for n in ("k_pages", "v_pages"))
    o2, l2 = torch.empty_like(o1), torch.empty_like(l1)
    ra.prefill(t["q"], k, v, t["qo_indptr"], t["scale"], out=o2, lse=l2)
    H.compare(o2, H.f64(o1), l2, H.f64(l1))


# ------------------------------------------------------------------------------------------- as an engine uses them

class Engine:
    """A model of one layer whose rows are given: requests, their tables and a pool of pages."""

    def __init__(self, batch, page, pool, fp8, seed=71):
        self.page, self.hq, self.hkv, self.fp8 = page, 16, 2, fp8
        kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
        self.pools = [torch.zeros((pool, page, 2, 128), device=DEV).to(kind) for _ in range(2)]
        self.scales = [dev(np.array([0.01, 0.013]), torch.float32), dev(np.array([0.012, 0.011]), torch.float32)]
        self.free = dev(np.random.default_rng(seed).permutation(pool))
        self.used, self.lens = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.table = torch.full((batch, 40), -1, dtype=torch.int32, device=DEV)
        self.freq = dev(1e6 ** (-np.arange(64) / 64), torch.float32)
        self.axes = dev(np.repeat([0, 1, 2], [16, 24, 24]))

    def map(self, new, rows, out=None):
        return ra.map_slots(self.lens, new, self.free, self.used, self.table, self.page, self.pools[0].shape[0], rows,
                            kv_lens_out=self.lens, free_used_out=self.used, **(out or {}))

    def turn(self, m, qkv, q_out=None, k_out=None):
        q, k, v = qkv[:, :16], qkv[:, 16:18], qkv[:, 18:]
        pos = m.positions.expand(3, -1)
        if self.fp8:
            return ra.rope_append_kv_fp8(q, k, v, pos, self.freq, m.slot_map, *self.pools, *self.scales, self.axes,
                                         q_out=q_out, k_out=k_out)
        return ra.rope_append_kv(q, k, v, pos, self.freq, m.slot_map, *self.pools, self.axes, q_out=q_out, k_out=k_out)

    def extend(self, m, q):
        args = (m.qo_indptr, *self.pools, *(self.scales if self.fp8 else []), self.table, m.kv_lens, 128 ** -0.5)
        return (ra.extend_fp8 if self.fp8 else ra.extend)(q, *args)

    def decode(self, m, q, out=None):
        args = (*self.pools, *(self.scales if self.fp8 else []), self.table, m.kv_lens, 128 ** -0.5)
        return (ra.decode_fp8 if self.fp8 else ra.decode)(q, *args, out=out)


@pytest.mark.parametrize("fp8", [False, True])
def test_turns_of_an_engine(fp8):
    """Prompts, a further turn and decode steps through map_slots, rope_append_kv, prefill, extend and decode equal
    attention over all rows so far, turned and attended to in 64 bits."""
    lens = [[70, 5, 130, 0], [30, 64, 1, 9], [1, 1, 1, 1], [1, 1, 1, 1]]
    e = Engine(4, 16, 200, fp8)
    held = [[] for _ in range(4)]                      # rows of each request so far
    for turn, new in enumerate(lens):
        total = sum(new)
        qkv = rand(80 + turn, total + 3, 20, 128)
        m = e.map(dev(np.array(new)), total + 3)
        k_rows = torch.zeros((total + 3, 2, 128), dtype=torch.bfloat16, device=DEV)
        q = e.turn(m, qkv, k_out=k_rows)
        if turn == 0:
            out = ra.prefill(q, k_rows, qkv[:, 18:], m.qo_indptr, 128 ** -0.5)[:total]
        elif turn == 1:
            out = e.extend(m, q)[:total]
        else:
            out = e.decode(m, q[:4])
        ra.check_device_errors()
        assert m.kv_lens.tolist() == [sum(x[b] for x in lens[:turn + 1]) for b in range(4)]
        rows = H.f64(qkv)
        at = 0
        for b, n in enumerate(new):
            held[b] += list(rows[at:at + n])
            if n:
                x = np.stack(held[b])
                pos = np.arange(len(x))[None].repeat(3, 0)
                freq, axes = e.freq.cpu().numpy(), e.axes.cpu().numpy()
                ref, _, _ = step.prefill(step.rope(x[:, :16], pos, freq, axes), step.rope(x[:, 16:18], pos, freq, axes),
                                         x[:, 18:], [0, len(x)], 128 ** -0.5)
                got = H.f64(out[at:at + n])
                # (bf16 rows of q and k: 2^-8 of each product's factors on top of what attention rounds; FP8 pages
                # 2^-4: a relative error of the whole, where the average of n values falls with their errors)
                rel = np.linalg.norm(got - ref[-n:]) / np.linalg.norm(ref[-n:])
                first_bf16 = not fp8 or turn == 0
                assert rel <= (2.0 ** -6 if first_bf16 else 2.0 ** -3), (turn, b, rel)
            at += n


@pytest.mark.parametrize("fp8", [False, True])
def test_captured_decode_steps_replay(fp8):
    """A decode step (map_slots in place, rope_append_kv, decode) captured once and replayed: each replay takes the
    requests one token further, with the results of eager steps, which run between the replays."""
    batch = 6
    a, b = Engine(batch, 8, 300, fp8), Engine(batch, 8, 300, fp8)
    first = np.array([9, 16, 1, 40, 7, 8])
    for e in (a, b):
        m = e.map(dev(first), int(first.sum()))
        e.turn(m, rand(90, int(first.sum()), 20, 128))
    one = dev(np.ones(batch))
    s = torch.cuda.Stream()
    ra.reserve_workspace(ra.decode_workspace_size(batch, 16, 2, 40, 8), stream=s)
    qkv = rand(91, batch + 2, 20, 128)                 # padded to a captured size
    got = {"slot_map": torch.zeros(batch + 2, dtype=torch.int64, device=DEV),
           "positions": torch.zeros(batch + 2, dtype=torch.int32, device=DEV),
           "qo_indptr": torch.zeros(batch + 1, dtype=torch.int32, device=DEV)}
    q, out = torch.zeros((batch + 2, 16, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((batch, 16, 128), dtype=torch.bfloat16, device=DEV)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        m = a.map(one, None, got)
        a.turn(m, qkv, q_out=q)
        a.decode(m, q[:batch], out=out)
    torch.cuda.synchronize()
    assert a.lens.tolist() == first.tolist(), "capturing runs nothing"
    for rep in range(20):                              # over page borders
        rows = rand(100 + rep, batch + 2, 20, 128)
        qkv.copy_(rows)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        mb = b.map(one, batch + 2)
        want = b.decode(mb, b.turn(mb, rows)[:batch])
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(got["slot_map"], mb.slot_map), rep
        assert torch.equal(a.lens, b.lens) and torch.equal(a.table, b.table) and torch.equal(a.used, b.used)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a.pools, b.pools))
    ra.check_device_errors(s)
    ra.check_device_errors()


def test_prefill_captured_and_on_another_stream():
    c = prompts(95, [200, 31, 77], 8, 2)
    ptr, s = dev(c["indptr"]), torch.cuda.Stream()
    out, lse = torch.zeros_like(c["q"]), torch.zeros((c["rows"], 8), device=DEV)
    ra.reserve_workspace(0, stream=s)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        ra.prefill(c["q"], c["k"], c["v"], ptr, 128 ** -0.5, out=out, lse=lse)
    for rep in range(4):
        c["q"].copy_(rand(200 + rep, *c["q"].shape))
        ptr.copy_(dev(np.array([[0, 200, 231, 308], [0, 0, 308, 308], [0, 100, 101, 250], [0, 1, 2, 3]][rep])))
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want, want_lse = torch.zeros_like(out), torch.zeros_like(lse)
        ra.prefill(c["q"], c["k"], c["v"], ptr, 128 ** -0.5, out=want, lse=want_lse)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse[:int(ptr[-1])], want_lse[:int(ptr[-1])]), rep


def test_views_describe_tensors():
    base = torch.zeros(6, 5, 4, 3, device=DEV)
    for t in (base, base[1:, ::2], base.permute(3, 1, 0, 2), base[2, 3], base[0, 0, 0, 1:], base[0, 0, 0, 0], base[:0],
              base[:, :1].expand(6, 9, 4, 3), base.to(torch.bfloat16), base.to(torch.int32), base.to(torch.int64),
              base.to(torch.float8_e4m3fn), base.to(torch.float16)):
        v, n = ra.view(t), t.dim()
        dtype = {torch.float32: ra.RL_F32, torch.bfloat16: ra.RL_BF16, torch.int32: ra.RL_I32, torch.int64: ra.RL_I64,
                 torch.float8_e4m3fn: ra.RL_FP8_E4M3}.get(t.dtype, 0)
        assert (v.data or 0, v.dtype, v.ndim) == (t.data_ptr(), dtype, n)
        assert list(v.shape) == [*t.shape] + [0] * (4 - n) and list(v.strides) == [*t.stride()] + [0] * (4 - n)
    with pytest.raises(ValueError, match="at most 4"):
        ra.view(base[None])
