"""The step calls refuse bad arguments before touching the GPU (CPU only; no compute calls)."""

import ctypes

import pytest

from paper_2609_08368_amd import rl_attn as ra
from tests.test_abi import FAKE, fake

I32, I64, F32, BF16, FP8 = ra.RL_I32, ra.RL_I64, ra.RL_F32, ra.RL_BF16, ra.RL_FP8_E4M3


def ref(x):
    return ctypes.byref(x) if isinstance(x, ctypes.Structure) else x


def refused(call, args, status, needle):
    rc = call(*(ref(a) for a in args.values()), None)
    assert ra.STATUS[rc] == status, (ra.STATUS[rc], ra.last_error())
    assert needle in ra.last_error(), ra.last_error()


def opts(**kw):
    o = ra.RlRopeOpts()
    for k, v in kw.items():
        setattr(o, k, v)
    return o


def with_reserved():
    o = ra.RlRopeOpts()
    o.reserved[5] = 1
    return o


def map_args(B=3, T=10, **kw):
    a = dict(kv=fake([B], I32), new=fake([B], I32), free=fake([20], I32), used=fake([1], I32), delta=None, page=16,
             pages=30, table=fake([B, 4], I32), kv_out=fake([B], I32), used_out=fake([1], I32), ptr=fake([B + 1], I32),
             slots=fake([T], I64), pos=fake([T], I32))
    return {**a, **kw}


@pytest.mark.parametrize("change,status,needle", [
    (dict(kv=None), "RL_ERR_INVALID_ARG", "kv_lens is NULL"),
    (dict(kv=fake([3, 1], I32)), "RL_ERR_SHAPE", "kv_lens must have 1"),
    (dict(new=fake([4], I32)), "RL_ERR_SHAPE", "new_lens must have 3"),
    (dict(new=fake([3], I64)), "RL_ERR_DTYPE", "new_lens must be int32 (got int64)"),
    (dict(free=fake([20], F32)), "RL_ERR_DTYPE", "free_pages"),
    (dict(free=fake([20], I32, ptr=0)), "RL_ERR_INVALID_ARG", "free_pages.data"),
    (dict(used=fake([2], I32)), "RL_ERR_SHAPE", "free_used"),
    (dict(delta=fake([2], I32)), "RL_ERR_SHAPE", "pos_delta"),
    (dict(page=24), "RL_ERR_UNSUPPORTED", "page size"),
    (dict(page=256), "RL_ERR_UNSUPPORTED", "page size"),
    (dict(pages=-1), "RL_ERR_INVALID_ARG", "num_pages"),
    (dict(pages=1 << 31), "RL_ERR_UNSUPPORTED", "too large"),
    (dict(table=fake([2, 4], I32)), "RL_ERR_SHAPE", "block_table.shape[0]"),
    (dict(table=fake([3, 1 << 24], I32)), "RL_ERR_UNSUPPORTED", "too large"),
    (dict(table=fake([3, 4], I32, strides=[0, 1])), "RL_ERR_UNSUPPORTED", "block_table"),
    (dict(table=fake([3, 4], I32, strides=[4, 0])), "RL_ERR_UNSUPPORTED", "block_table"),
    (dict(kv_out=fake([3], I32, strides=[0])), "RL_ERR_UNSUPPORTED", "kv_lens_out: stride"),
    (dict(kv_out=fake([3], I32, strides=[2])), "RL_ERR_UNSUPPORTED", "kv_lens_out must be kv_lens or not overlap it"),
    (dict(kv_out=fake([3], I32, ptr=FAKE + 4)), "RL_ERR_UNSUPPORTED", "kv_lens_out must be kv_lens or not overlap it"),
    (dict(kv_out=fake([3], I32, ptr=FAKE - 8)), "RL_ERR_UNSUPPORTED", "kv_lens_out must be kv_lens or not overlap it"),
    (dict(ptr=fake([3], I32)), "RL_ERR_SHAPE", "qo_indptr must have 4"),
    (dict(slots=fake([10], I32)), "RL_ERR_DTYPE", "slot_map must be int64"),
    (dict(slots=fake([1 << 31], I64)), "RL_ERR_UNSUPPORTED", "too long"),
    (dict(pos=fake([9], I32)), "RL_ERR_SHAPE", "positions must have 10"),
    (dict(pos=fake([10], I32, strides=[-1])), "RL_ERR_UNSUPPORTED", "positions"),
])
def test_map_slots_refuses(change, status, needle):
    refused(ra.lib().rl_attn_map_slots, map_args(**change), status, needle)


@pytest.mark.parametrize("change", [
    dict(kv_out=fake([3], I32, ptr=FAKE + 12)), dict(kv_out=fake([3], I32, ptr=FAKE - 12)),
    dict(kv=fake([3], I32, strides=[2]), kv_out=fake([3], I32, strides=[2], ptr=FAKE + 4)),
    dict(kv=fake([3], I32, strides=[2]), kv_out=fake([3], I32, strides=[2]))])
def test_map_slots_takes_lengths_beside_each_other(change):
    """(as far as the check of its last argument)"""
    refused(ra.lib().rl_attn_map_slots, map_args(**change, pos=fake([9], I32)), "RL_ERR_SHAPE", "positions must have 10")


def rope_args(T=10, hq=8, hkv=2, F=64, **kw):
    a = dict(q=fake([T, hq, 128], BF16), k=fake([T, hkv, 128], BF16), pos=fake([3, T], I32), freq=fake([F], F32),
             axes=fake([F], I32), opts=None, q_out=fake([T, hq, 128], BF16), k_out=fake([T, hkv, 128], BF16))
    return {**a, **kw}


ROPE_REFUSALS = [
    (dict(q=None), "RL_ERR_INVALID_ARG", "q is NULL"),
    (dict(q=fake([10, 8, 64], BF16)), "RL_ERR_UNSUPPORTED", "head dimension must be 128"),
    (dict(q=fake([10, 8, 128], F32)), "RL_ERR_DTYPE", "q must be bf16"),
    (dict(q=fake([10, 8, 128], BF16, ptr=FAKE + 8)), "RL_ERR_UNSUPPORTED", "aligned"),
    (dict(q_out=None), "RL_ERR_INVALID_ARG", "q_out is NULL"),
    (dict(q_out=fake([10, 7, 128], BF16)), "RL_ERR_SHAPE", "q_out must be [10, 8, 128]"),
    (dict(q_out=fake([10, 8, 128], BF16, strides=[1024, 0, 1])), "RL_ERR_UNSUPPORTED", "must not overlap"),
    (dict(q_out=fake([10, 8, 128], BF16, strides=[256, 128, 1])), "RL_ERR_UNSUPPORTED", "must not overlap"),
    (dict(q_out=fake([10, 8, 128], BF16, strides=[128, 1272, 1])), "RL_ERR_UNSUPPORTED", "must not overlap"),
    (dict(k_out=fake([9, 2, 128], BF16)), "RL_ERR_SHAPE", "k_out"),
    (dict(pos=fake([10], I32)), "RL_ERR_SHAPE", "positions must have 2"),
    (dict(pos=fake([3, 9], I32)), "RL_ERR_SHAPE", "positions must be"),
    (dict(pos=fake([3, 10], I64)), "RL_ERR_DTYPE", "positions must be int32"),
    (dict(axes=None), "RL_ERR_INVALID_ARG", "axes is NULL"),
    (dict(axes=fake([32], I32)), "RL_ERR_SHAPE", "axes must have 64"),
    (dict(freq=fake([60], F32), axes=fake([60], I32)), "RL_ERR_UNSUPPORTED", "multiple of 8"),
    (dict(freq=fake([72], F32), axes=fake([72], I32)), "RL_ERR_UNSUPPORTED", "8 to 64"),
    (dict(freq=fake([0], F32), axes=fake([0], I32)), "RL_ERR_UNSUPPORTED", "8 to 64"),
    (dict(opts=opts(interleaved=2)), "RL_ERR_INVALID_ARG", "interleaved"),
    (dict(opts=opts(inverse=-1)), "RL_ERR_INVALID_ARG", "inverse"),
    (dict(opts=with_reserved()), "RL_ERR_INVALID_ARG", "reserved[5]"),
]


@pytest.mark.parametrize("change,status,needle", ROPE_REFUSALS + [
    (dict(k=None), "RL_ERR_INVALID_ARG", "k is NULL"), (dict(k_out=None), "RL_ERR_INVALID_ARG", "k_out is NULL")])
def test_rope_refuses(change, status, needle):
    refused(ra.lib().rl_attn_rope, rope_args(**change), status, needle)


def append_args(fp8, T=10, hq=8, hkv=2, **kw):
    r = rope_args(T, hq, hkv)
    pages = [fake([30, 16, hkv, 128], FP8 if fp8 else BF16) for _ in range(2)]
    a = dict(q=r["q"], k=r["k"], v=fake([T, hkv, 128], BF16), pos=r["pos"], freq=r["freq"], axes=r["axes"], opts=None,
             slots=fake([T], I64), q_out=r["q_out"], k_out=None, kp=pages[0], vp=pages[1])
    if fp8:
        a.update(ks=fake([hkv], F32), vs=fake([hkv], F32))
    return {**a, **kw}


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("change,status,needle", ROPE_REFUSALS + [
    (dict(k=None), "RL_ERR_INVALID_ARG", "k_new is NULL"),
    (dict(v=None), "RL_ERR_INVALID_ARG", "v_new is NULL"),
    (dict(v=fake([10, 3, 128], BF16)), "RL_ERR_SHAPE", "v_new"),
    (dict(slots=None), "RL_ERR_INVALID_ARG", "slot_map is NULL"),
    (dict(slots=fake([10], I32)), "RL_ERR_DTYPE", "slot_map must be int64"),
    (dict(slots=fake([11], I64)), "RL_ERR_SHAPE", "slot_map must have 10"),
    (dict(opts=opts(inverse=1)), "RL_ERR_INVALID_ARG", "not appended"),
    (dict(kp=fake([30, 16, 2, 128], F32)), "RL_ERR_DTYPE", "k_pages must be"),
    (dict(vp=None), "RL_ERR_INVALID_ARG", "v_pages is NULL"),
    (dict(vp=fake([30, 32, 2, 128], BF16), kp=fake([30, 16, 2, 128], BF16)), "RL_ERR_", ""),
])
def test_rope_append_refuses(change, status, needle, fp8):
    call = ra.lib().rl_attn_rope_append_kv_fp8 if fp8 else ra.lib().rl_attn_rope_append_kv
    args = append_args(fp8, **change)
    if status == "RL_ERR_":                        # (the pools' shapes differ: for FP8 their type is refused first)
        status, needle = ("RL_ERR_DTYPE", "k_pages") if fp8 else ("RL_ERR_SHAPE", "shapes differ")
    refused(call, args, status, needle)


def test_rope_append_checks_pools_against_rows():
    for fp8, call in ((False, ra.lib().rl_attn_rope_append_kv), (True, ra.lib().rl_attn_rope_append_kv_fp8)):
        kind = FP8 if fp8 else BF16
        three = dict(kp=fake([30, 16, 3, 128], kind), vp=fake([30, 16, 3, 128], kind))
        if fp8:
            three.update(ks=fake([3], F32), vs=fake([3], F32))
        refused(call, append_args(fp8, **three), "RL_ERR_SHAPE", "KV heads")
    refused(ra.lib().rl_attn_rope_append_kv_fp8, append_args(True, ks=fake([1], F32)), "RL_ERR_SHAPE", "k_scale")
    refused(ra.lib().rl_attn_rope_append_kv_fp8, append_args(True, vs=None), "RL_ERR_INVALID_ARG", "v_scale is NULL")


def prefill_args(T=10, hq=8, hkv=2, B=3, scale=0.1, **kw):
    a = dict(q=fake([T, hq, 128], BF16), k=fake([T, hkv, 128], BF16), v=fake([T, hkv, 128], BF16),
             ptr=fake([B + 1], I32), scale=ctypes.c_float(scale), out=fake([T, hq, 128], BF16), lse=None)
    return {**a, **kw}


@pytest.mark.parametrize("change,status,needle", [
    (dict(q=None), "RL_ERR_INVALID_ARG", "q is NULL"),
    (dict(q=fake([10, 8, 64], BF16)), "RL_ERR_UNSUPPORTED", "head dimension"),
    (dict(k=fake([10, 3, 128], BF16)), "RL_ERR_SHAPE", "multiple of KV heads"),
    (dict(k=fake([10, 0, 128], BF16)), "RL_ERR_SHAPE", "multiple of KV heads"),
    (dict(k=fake([11, 2, 128], BF16)), "RL_ERR_SHAPE", "k must be [10, 2, 128]"),
    (dict(v=fake([10, 4, 128], BF16)), "RL_ERR_SHAPE", "v must be [10, 2, 128]"),
    (dict(v=fake([10, 2, 128], FP8)), "RL_ERR_DTYPE", "v must be bf16"),
    (dict(k=fake([10, 2, 128], BF16, strides=[1 << 24, 128, 1])), "RL_ERR_UNSUPPORTED", "2^24"),
    (dict(ptr=fake([0], I32)), "RL_ERR_SHAPE", "batch + 1"),
    (dict(ptr=fake([4], I64)), "RL_ERR_DTYPE", "seq_indptr must be int32"),
    (dict(ptr=None), "RL_ERR_INVALID_ARG", "seq_indptr is NULL"),
    (dict(scale=0.0), "RL_ERR_INVALID_ARG", "scale"),
    (dict(scale=float("nan")), "RL_ERR_INVALID_ARG", "scale"),
    (dict(out=fake([9, 8, 128], BF16)), "RL_ERR_SHAPE", "out shape"),
    (dict(out=fake([10, 8, 128], I32)), "RL_ERR_DTYPE", "out must be bf16 or f32"),
    (dict(lse=fake([10, 7], F32)), "RL_ERR_SHAPE", "lse_out"),
    (dict(T=1 << 26, hq=64, hkv=8), "RL_ERR_UNSUPPORTED", "rows times heads"),
])
def test_prefill_refuses(change, status, needle):
    refused(ra.lib().rl_attn_prefill, prefill_args(**change), status, needle)


def test_calls_of_nothing_are_no_ops():
    lib = ra.lib()
    for call, args in ((lib.rl_attn_rope, rope_args(T=0)), (lib.rl_attn_rope_append_kv, append_args(False, T=0)),
                       (lib.rl_attn_prefill, prefill_args(T=0)), (lib.rl_attn_prefill, prefill_args(B=0))):
        assert call(*(ref(a) for a in args.values()), None) == 0, ra.last_error()


def test_a_tensor_is_described_or_refused():
    """(on a GPU too, in the tests that run there)"""
    import torch

    assert ra.view(None) is None
    with pytest.raises(ValueError, match="tensor on cpu: .* current device"):
        ra.view(torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError, match="expected a tensor or None, got list"):
        ra.view([1, 2])
