"""The step's calls at sizes that take other routes than the small ones, on the GPU: slot maps of more than 4096 requests
(several passes), and more than 256 prompts (units in the order of the rows)."""

import numpy as np
import pytest
import torch

from oracle import step
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_step import bits, check_map, check_rows, map_case, prompts, run_prefill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch", [4095, 4096, 4097, 9001])
def test_map_of_several_passes(batch, in_place):
    H.say(f"map {batch} in_place={in_place}")
    for new in (1, 7):
        check_map(map_case(batch + new, batch, 40, new, 8, 5, new_lo=int(new == 1)), in_place)


@pytest.mark.parametrize("change", [
    lambda c: c["kv_lens"].__setitem__(4100, -1), lambda c: c["new_lens"].__setitem__(4100, 10 ** 9),
    lambda c: c.update(rows=100), lambda c: c.update(rows=c["rows"] - 1), lambda c: c.update(rows=c["rows"] // 2),
    lambda c: c.update(free_pages=c["free_pages"][:60]), lambda c: c.update(free_pages=c["free_pages"][:-12]),
    lambda c: c["new_lens"].__setitem__(slice(4096, None), 0), lambda c: c["new_lens"].__setitem__(slice(0, 4096), 0),
    lambda c: c["block_table"].__setitem__((slice(None), slice(0, 9)), -1)], ids=range(10))
def test_map_of_several_passes_refuses_and_reports(change):
    """A request that is served last, in the first pass, on a pass's border or in the last one."""
    for in_place in (False, True):
        c = map_case(12, 8500, 40, 7, 8)
        change(c)
        check_map(c, in_place)


@pytest.mark.parametrize("lens,hq,hkv", [
    ([3] * 257, 8, 2), ([1, 0, 70, 2] * 90, 4, 1), ([0] * 300 + [130] + [5] * 40, 8, 8), ([40, 65, 1] * 150, 32, 8),
    ([0] * 400, 8, 2)], ids=["257x3", "360", "341", "450", "none"])
def test_prefill_of_many_prompts(lens, hq, hkv):
    H.say(f"prefill {len(lens)} prompts {hq}/{hkv}")
    c = prompts(len(lens), lens, hq, hkv, pad=6)
    n = int(c["indptr"][-1])
    ref = step.prefill(bits(c["q"]), bits(c["k"]), bits(c["v"]), c["indptr"], 128 ** -0.5)
    for dtype in (torch.bfloat16, torch.float32):
        out, lse = run_prefill(c, dtype)
        check_rows(out[:n], lse[:n], *(r[:n] for r in ref), dtype == torch.float32)
        assert torch.isnan(out[n:]).all() and torch.isnan(lse[n:]).all(), "rows of no prompt are left as they were"
    again, _ = run_prefill(c, torch.float32)
    assert torch.equal(again[:n], out[:n])
    ra.check_device_errors()


def test_prefill_of_many_prompts_clamps_and_reports_bounds():
    """Bounds that fall, start above zero and end past the rows, among 300 prompts: the sound prompts' rows are right."""
    lens = [4] * 300
    c = prompts(3, lens, 8, 2)
    c["indptr"] = c["indptr"].copy()
    c["indptr"][0], c["indptr"][150], c["indptr"][300] = 2, 590, 5000
    out, lse = run_prefill(c)
    with pytest.raises(ra.RlAttnError) as e:
        ra.check_device_errors()
    assert "indptr-invalid" in str(e.value)
    assert torch.isnan(out[:2]).all()
    # (prompt 149 has no rows left; prompt 150 has those from 590 on, with 148's behind them)
    sound = np.concatenate([[2], np.arange(4, 593, 4), np.arange(604, 1197, 4)])
    ref = step.prefill(bits(c["q"]), bits(c["k"]), bits(c["v"]), sound, 128 ** -0.5)
    rows = [*range(2, 588), *range(604, 1196)]
    check_rows(out[rows], lse[rows], *(r[rows] for r in ref))


@pytest.mark.parametrize("hq,hkv", [(8, 2), (96, 8), (96, 96)])
def test_prefill_keeps_the_bits_of_rows_that_see_no_odd_value(hq, hkv):
    """Infinities and NaN in one prompt's keys or values: the other prompts' rows keep their bits, and so do the rows of
    the same prompt's earlier tiles; the rows that see them are not numbers (their log-sum-exp is where a key is odd)."""
    lens = [150, 411, 60]
    c = prompts(21, lens, hq, hkv, pad=5)
    out, lse = run_prefill(c)
    n, at = int(c["indptr"][-1]), 150 + 300
    for bad in (float("nan"), float("inf")):
        for name in ("k", "v"):
            d = dict(c, **{name: c[name].clone()})
            d[name][at] = bad
            o, l = run_prefill(d)
            same = [*range(150), *range(150, 150 + 300 - 256), *range(561, n)]
            assert torch.equal(o[same], out[same]) and torch.equal(l[same], lse[same]), (name, bad)
            sees = slice(at, 561)
            assert not torch.isfinite(o[sees]).any() if np.isnan(bad) or name == "v" else True, (name, bad)
            if name == "k" and np.isnan(bad):
                assert torch.isnan(l[sees]).all()
            if name == "v":
                assert torch.equal(l[sees].isfinite(), torch.ones_like(l[sees], dtype=torch.bool))
            assert torch.isfinite(o[150:at]).all() and torch.isfinite(l[150:at]).all()
