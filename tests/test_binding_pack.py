"""The binding describes tensors by a compiled module where there is one that loads, and by itself where there is not."""

import sys
import warnings

import pytest
import torch

from paper_2609_08368_amd import rl_attn as ra


@pytest.fixture
def fresh(monkeypatch):
    """The binding as after its import, before a first call."""
    monkeypatch.setattr(ra, "_arg", ra._first_arg)
    return monkeypatch


def refusals():
    assert ra.view(None) is None
    with pytest.raises(ValueError, match="tensor on cpu: .* current device"):
        ra.view(torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError, match="expected a tensor or None, got list"):
        ra.view([1, 2])


def test_the_module_is_found_at_the_first_call(fresh):
    refusals()
    from paper_2609_08368_amd import _pack

    assert ra._arg is _pack.arg


def test_a_module_built_after_the_import_is_found(fresh, tmp_path):
    built, fresh_path = ra._PACK_PATH, str(tmp_path / "_pack.so")
    fresh.setattr(ra, "_PACK_PATH", fresh_path)
    refusals()
    assert ra._arg is ra._first_arg, "not built: looked for again at the next call"
    fresh.setattr(ra, "_PACK_PATH", built)
    refusals()
    assert ra._arg is not ra._first_arg


def test_a_module_that_does_not_load_is_named_once(fresh):
    fresh.setitem(sys.modules, "paper_2609_08368_amd._pack", None)          # (the import raises ImportError)
    fresh.delattr("paper_2609_08368_amd._pack", raising=False)
    with pytest.warns(RuntimeWarning, match="_pack.so does not load"):
        refusals()
    assert ra._arg is ra._describe
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        refusals()


@pytest.mark.gpu
def test_both_describe_tensors_alike():
    from paper_2609_08368_amd import _pack

    base = torch.zeros(6, 5, 4, 3, device="cuda:0")
    for t in (base, base[1:, ::2], base.permute(3, 1, 0, 2), base[2, 3], base[0, 0, 0, 1:], base[0, 0, 0, 0], base[:0],
              base[:, :1].expand(6, 9, 4, 3), base.to(torch.bfloat16), base.to(torch.int32), base.to(torch.int64),
              base.to(torch.float8_e4m3fn), base.to(torch.float16), torch.empty(0, 7, device="cuda:0")):
        assert ra._describe(t) == _pack.arg(t)
    for f in (ra._describe, _pack.arg):
        with pytest.raises(ValueError, match="at most 4"):
            f(base[None])
    assert ra._describe(None) is None and _pack.arg(None) is None


@pytest.mark.gpu
def test_calls_without_the_module(monkeypatch):
    q, k, v = (torch.randn(20, h, 128, device="cuda:0").to(torch.bfloat16) for h in (8, 2, 2))
    ptr = torch.tensor([0, 13, 20], dtype=torch.int32, device="cuda:0")
    want = ra.prefill(q, k, v, ptr, 0.1)
    monkeypatch.setattr(ra, "_arg", ra._describe)
    assert torch.equal(ra.prefill(q, k, v, ptr, 0.1), want)
