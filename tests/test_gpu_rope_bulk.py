"""Rotary rows of more than 8192 eights of head rows (16 head rows a wave, stored nontemporally) on the GPU: against the
definition, in place, and with the bits that the same rows have in calls of a few hundred."""

import numpy as np
import pytest
import torch

from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_step import DEV, append_case, axes_of, check_turned, dev, rope_args, rope_case, run_append

pytestmark = pytest.mark.gpu


def halves(c, n):
    """The case's first rows (few enough for the other kernel), as often as it takes."""
    return [slice(at, min(at + n, len(c["q"]))) for at in range(0, len(c["q"]), n)]


# eights of head rows: with an odd number of them a row's last wave has one; heads that are no multiple of 8 end inside
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size", [(1100, 64, 8, 64), (1025, 56, 8, 48), (2800, 13, 5, 64), (8200, 1, 0, 8), (4200, 7, 4, 32)],
                         ids=str)
def test_rope_of_many_rows(size, interleaved):
    rows, hq, hkv, freqs = size
    assert rows * ((hq + hkv + 7) // 8) > 8192
    H.say(f"rope {size} interleaved={interleaved}")
    c = rope_case(rows, rows, hq, max(hkv, 1), freqs, axes_of(("text", "blocks", "cycle")[rows % 3], freqs))
    (pos, freq), axes = rope_args(c)
    k = c["k"] if hkv else None
    for inverse in (False, True):
        kw = dict(interleaved=interleaved, inverse=inverse)
        got = ra.rope(c["q"], k, pos, freq, axes, **kw)
        check_turned(got[0], c["q"], c, interleaved, inverse, what="q")
        if hkv:
            check_turned(got[1], k, c, interleaved, inverse, what="k")
        # in place in a fused buffer, whose other rows stay as they are, and in the small calls' kernel: the same bits
        fused = torch.cat((c["q"], c["k"], c["v"]), dim=1)
        mine = fused.clone()
        views = [mine[:, :hq], mine[:, hq:hq + hkv] if hkv else None]
        ra.rope(*views, pos, freq, axes, q_out=views[0], k_out=views[1], **kw)
        for i, x in enumerate(got):
            assert x is None or torch.equal(views[i], x)
        assert torch.equal(mine[:, hq + hkv:], fused[:, hq + hkv:])
        for part in halves(c, 300):
            few = ra.rope(c["q"][part], None if k is None else k[part], pos[:, part], freq, axes, **kw)
            assert all(x is None or torch.equal(x, y[part]) for x, y in zip(few, got))
    ra.check_device_errors()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("size", [(1000, 64, 8, 64, 64, 39), (1200, 48, 4, 40, 16, 7), (4000, 9, 3, 64, 8, 200)], ids=str)
def test_rope_append_of_many_rows(size, fp8):
    rows, hq, hkv, freqs, page, pad = size
    assert (rows + pad) * ((hq + 2 * hkv + 7) // 8) > 8192
    interleaved = rows % 16 == 0
    H.say(f"rope append {size} fp8={fp8}")
    c = append_case(rows, rows, hq, hkv, freqs, axes_of("cycle", freqs), page, fp8, pad)
    c["slots"][5] = -7                                     # rows without a slot between others, and at the end
    c["slots"][rows - 2] = -1
    real = np.flatnonzero(c["slots"] >= 0)
    pools = [p.clone() for p in c["pools"]]
    marks = [torch.full_like(c[n], 7.0) for n in "qk"]
    q, k = (m.clone() for m in marks)
    run_append(c, interleaved, q, k, pools)
    ra.check_device_errors()
    check_turned(q, c["q"], c, interleaved, rows=real, what="q")
    check_turned(k, c["k"], c, interleaved, rows=real, what="k")
    none = torch.from_numpy(np.flatnonzero(c["slots"] < 0)).to(DEV)
    assert torch.equal(q[none], marks[0][none]) and torch.equal(k[none], marks[1][none])
    # the small calls' kernel, some rows at a time: the same rows and pages
    (pos, freq), axes = rope_args(c)
    slots = dev(c["slots"], torch.int64)
    call = ra.rope_append_kv_fp8 if fp8 else ra.rope_append_kv
    few, q2, k2 = [p.clone() for p in c["pools"]], *(m.clone() for m in marks)
    for part in halves(c, 250):
        call(c["q"][part], c["k"][part], c["v"][part], pos[:, part], freq, slots[part], *few, *c["scales"], axes,
             interleaved=interleaved, q_out=q2[part], k_out=k2[part])
    assert torch.equal(q, q2) and torch.equal(k, k2)
    for a, b in zip(pools, few):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    if not fp8:
        flat = [p.view(-1, hkv, 128) for p in pools]
        at = slots[torch.from_numpy(real).to(DEV)]
        assert torch.equal(flat[0][at], k[real]) and torch.equal(flat[1][at], c["v"][real])
    # in place in a fused buffer
    fused = torch.cat((c["q"], c["k"], c["v"]), dim=1)
    views = [fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]]
    again = [p.clone() for p in c["pools"]]
    call(*views, pos, freq, slots, *again, *c["scales"], axes, interleaved=interleaved, q_out=views[0], k_out=views[1])
    assert torch.equal(views[0][real], q[real]) and torch.equal(views[1][real], k[real])
    assert torch.equal(views[0][none], c["q"][none]) and torch.equal(views[2], c["v"])
    for a, b in zip(again, pools):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
