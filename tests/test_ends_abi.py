"""The calls at a step's ends refuse bad arguments before touching the GPU (CPU only; no compute calls)."""

import ctypes

import pytest

from paper_2609_08368_amd import rl_attn as ra
from tests.test_abi import FAKE, fake
from tests.test_step_abi import BF16, F32, FP8, I32, I64, opts, refused, with_reserved
from tests.test_step_overlap import ROWS, apart

EPS = ctypes.c_float(1e-6)


def refusals(call, make, cases):
    for change, status, needle in cases:
        refused(call, make(**change), status, needle)


# ---------------------------------------------------------------------------------------------- normed rotary rows

def norm_args(T=10, hq=8, hkv=2, F=64, **kw):
    a = dict(q=fake([T, hq, 128], BF16), k=fake([T, hkv, 128], BF16), qw=fake([128], BF16), kw=fake([128], BF16),
             eps=EPS, pos=fake([3, T], I32), freq=fake([F], F32), axes=fake([F], I32), opts=None,
             q_out=fake([T, hq, 128], BF16), k_out=fake([T, hkv, 128], BF16))
    return {**a, **kw}


NORM = [
    (dict(qw=None), "RL_ERR_INVALID_ARG", "q_weight is NULL"),
    (dict(qw=fake([64], BF16)), "RL_ERR_SHAPE", "q_weight must have 128"),
    (dict(qw=fake([8, 128], BF16)), "RL_ERR_SHAPE", "q_weight must have 1"),
    (dict(qw=fake([128], I32)), "RL_ERR_DTYPE", "q_weight must be bf16 or f32"),
    (dict(qw=fake([128], F32)), "RL_ERR_DTYPE", "must have one type"),
    (dict(kw=fake([128], F32)), "RL_ERR_DTYPE", "must have one type"),
    (dict(kw=None), "RL_ERR_INVALID_ARG", "k_weight is NULL"),
    (dict(kw=fake([128], BF16, strides=[2])), "RL_ERR_UNSUPPORTED", "stride must be 1"),
    (dict(kw=fake([128], BF16, ptr=FAKE + 8)), "RL_ERR_UNSUPPORTED", "aligned"),
    (dict(kw=fake([128], BF16, ptr=0)), "RL_ERR_INVALID_ARG", "k_weight.data"),
    (dict(eps=ctypes.c_float(0.0)), "RL_ERR_INVALID_ARG", "eps"),
    (dict(eps=ctypes.c_float(-1e-6)), "RL_ERR_INVALID_ARG", "eps"),
    (dict(eps=ctypes.c_float(1e-40)), "RL_ERR_INVALID_ARG", "eps"),
    (dict(eps=ctypes.c_float(float("nan"))), "RL_ERR_INVALID_ARG", "eps"),
    (dict(eps=ctypes.c_float(float("inf"))), "RL_ERR_INVALID_ARG", "eps"),
    (dict(q=None), "RL_ERR_INVALID_ARG", "q is NULL"),
    (dict(q=fake([10, 8, 64], BF16)), "RL_ERR_UNSUPPORTED", "head dimension must be 128"),
    (dict(q=fake([10, 8, 128], F32)), "RL_ERR_DTYPE", "q must be bf16"),
    (dict(pos=fake([3, 9], I32)), "RL_ERR_SHAPE", "positions must be"),
    (dict(axes=None), "RL_ERR_INVALID_ARG", "axes is NULL"),
    (dict(freq=fake([72], F32), axes=fake([72], I32)), "RL_ERR_UNSUPPORTED", "8 to 64"),
    (dict(opts=opts(inverse=1)), "RL_ERR_INVALID_ARG", "opts.inverse is for"),
    (dict(opts=opts(interleaved=2)), "RL_ERR_INVALID_ARG", "interleaved"),
    (dict(opts=with_reserved()), "RL_ERR_INVALID_ARG", "reserved[5]"),
]


def test_norm_rope_refuses():
    refusals(ra.lib().rl_attn_norm_rope, norm_args, NORM + [
        (dict(k=None, k_out=None), "RL_ERR_INVALID_ARG", "k_weight is given, but k is NULL"),
        (dict(k=None, kw=None), "RL_ERR_INVALID_ARG", "k is NULL"),
        (dict(q_out=fake([10, 7, 128], BF16)), "RL_ERR_SHAPE", "q_out must be [10, 8, 128]"),
        (dict(k_out=None), "RL_ERR_INVALID_ARG", "k_out is NULL")])
    for name, make, needle in [
            ("q_out", lambda a: fake([10, 8, 128], BF16, a["q"].data + ROWS), "q_out must be q or not overlap it"),
            ("k_out", lambda a: fake([10, 2, 128], BF16, a["q"].data), "k_out and q"),
            ("qw", lambda a: fake([128], BF16, a["q_out"].data + 79 * ROWS), "q_out and q_weight"),
            ("kw", lambda a: fake([128], BF16, a["k_out"].data), "k_out and k_weight")]:
        a = apart(norm_args())
        refused(ra.lib().rl_attn_norm_rope, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


@pytest.mark.parametrize("fp8", [False, True])
def test_norm_rope_append_refuses(fp8):
    def make(T=10, hq=8, hkv=2, **kw):
        a = norm_args(T, hq, hkv)
        pool = fake([6, 16, hkv, 128], FP8 if fp8 else BF16)
        a = dict(q=a["q"], k=a["k"], v=fake([T, hkv, 128], BF16), qw=a["qw"], kw=a["kw"], eps=EPS, pos=a["pos"],
                 freq=a["freq"], axes=a["axes"], opts=None, slots=fake([T], I64), q_out=a["q_out"], k_out=None,
                 kp=pool, vp=pool)
        if fp8:
            a.update(ks=fake([hkv], F32), vs=fake([hkv], F32))
        return {**a, **kw}

    call = ra.lib().rl_attn_norm_rope_append_kv_fp8 if fp8 else ra.lib().rl_attn_norm_rope_append_kv
    refusals(call, make, NORM + [
        (dict(k=None), "RL_ERR_INVALID_ARG", "k_new is NULL"), (dict(v=None), "RL_ERR_INVALID_ARG", "v_new is NULL"),
        (dict(slots=fake([10], I32)), "RL_ERR_DTYPE", "slot_map must be int64"),
        (dict(kp=fake([6, 16, 2, 128], F32)), "RL_ERR_DTYPE", "k_pages"),
        (dict(kp=fake([6, 16, 3, 128], FP8 if fp8 else BF16), vp=fake([6, 16, 3, 128], FP8 if fp8 else BF16),
              **(dict(ks=fake([3], F32), vs=fake([3], F32)) if fp8 else {})), "RL_ERR_SHAPE", "KV heads")])


def grad_args(T=10, hq=8, hkv=2, **kw):
    n = norm_args(T, hq, hkv)
    a = dict(gq=fake([T, hq, 128], BF16), gk=fake([T, hkv, 128], BF16),
             **{k: n[k] for k in ("q", "k", "qw", "kw", "eps", "pos", "freq", "axes", "opts")},
             dq=fake([T, hq, 128], BF16), dk=fake([T, hkv, 128], BF16), dqw=fake([128], F32), dkw=fake([128], F32))
    return {**a, **kw}


def test_norm_rope_backward_refuses():
    call = ra.lib().rl_attn_norm_rope_backward
    refusals(call, grad_args, NORM + [
        (dict(gq=None), "RL_ERR_INVALID_ARG", "dq_out is NULL"), (dict(gk=None), "RL_ERR_INVALID_ARG", "dk_out is NULL"),
        (dict(gq=fake([10, 8, 128], F32)), "RL_ERR_DTYPE", "dq_out must be bf16"),
        (dict(gk=fake([10, 3, 128], BF16)), "RL_ERR_SHAPE", "dk_out must be"),
        (dict(dq=None), "RL_ERR_INVALID_ARG", "dq is NULL"), (dict(dk=None), "RL_ERR_INVALID_ARG", "dk is NULL"),
        (dict(dqw=None), "RL_ERR_INVALID_ARG", "dq_weight is NULL"),
        (dict(dqw=fake([128], BF16)), "RL_ERR_DTYPE", "dq_weight must be f32"),
        (dict(dkw=fake([127], F32)), "RL_ERR_SHAPE", "dk_weight"),
        (dict(dkw=fake([128], F32, strides=[0])), "RL_ERR_UNSUPPORTED", "dk_weight"),
        (dict(k=None), "RL_ERR_INVALID_ARG", "k is NULL"),
        (dict(dq=fake([10, 8, 128], BF16, strides=[1024, 0, 1])), "RL_ERR_UNSUPPORTED", "must not overlap")])
    for name, make, needle in [
            ("dq", lambda a: fake([10, 8, 128], BF16, a["q"].data), "dq and q"),
            ("dq", lambda a: fake([10, 8, 128], BF16, a["gq"].data + ROWS), "dq must be dq_out or not overlap it"),
            ("dk", lambda a: fake([10, 2, 128], BF16, a["gq"].data), "dk and dq_out"),
            ("dk", lambda a: fake([10, 2, 128], BF16, a["dq"].data), "dq and dk"),
            ("dkw", lambda a: fake([128], F32, a["dqw"].data + 4), "dq_weight and dk_weight"),
            ("dkw", lambda a: fake([128], F32, a["k"].data), "dk_weight and k"),
            ("dqw", lambda a: fake([128], F32, a["qw"].data), "dq_weight and q_weight")]:
        a = apart(grad_args())
        refused(call, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


# --------------------------------------------------------------------------------------------- log probabilities

def lp_args(T=10, V=100, K=3, **kw):
    a = dict(x=fake([T, V], BF16), tok=fake([T], I64), scale=fake([T], F32), lp=fake([T], F32), ent=fake([T], F32),
             lse=fake([T], F32), ids=fake([T, K], I32), lps=fake([T, K], F32))
    return {**a, **kw}


LOGITS = [
    (dict(x=None), "RL_ERR_INVALID_ARG", "logits is NULL"),
    (dict(x=fake([10], BF16)), "RL_ERR_SHAPE", "logits must have 2"),
    (dict(x=fake([10, 100], FP8)), "RL_ERR_DTYPE", "logits must be bf16 or f32"),
    (dict(x=fake([10, 100], BF16, strides=[1, 10])), "RL_ERR_UNSUPPORTED", "last stride"),
    (dict(x=fake([10, 100], BF16, strides=[-100, 1])), "RL_ERR_UNSUPPORTED", "row stride"),
    (dict(x=fake([10, 100], BF16, ptr=FAKE + 1)), "RL_ERR_UNSUPPORTED", "aligned"),
    (dict(x=fake([10, 100], F32, ptr=FAKE + 2)), "RL_ERR_UNSUPPORTED", "aligned"),
    (dict(x=fake([10, 100], BF16, ptr=0)), "RL_ERR_INVALID_ARG", "logits.data"),
    (dict(x=fake([10, 0], BF16)), "RL_ERR_SHAPE", "at least one column"),
    (dict(x=fake([10, (1 << 21) + 1], BF16)), "RL_ERR_UNSUPPORTED", "too large"),
    (dict(tok=None), "RL_ERR_INVALID_ARG", "tokens is NULL"),
    (dict(tok=fake([9], I64)), "RL_ERR_SHAPE", "tokens must have 10"),
    (dict(tok=fake([10, 1], I64)), "RL_ERR_SHAPE", "tokens must have 1"),
    (dict(tok=fake([10], F32)), "RL_ERR_DTYPE", "tokens must be int32 or int64"),
    (dict(scale=fake([1], F32)), "RL_ERR_SHAPE", "row_scale must have 10"),
    (dict(scale=fake([10], BF16)), "RL_ERR_DTYPE", "row_scale must be f32"),
]


def test_token_logprobs_refuses():
    call = ra.lib().rl_attn_token_logprobs
    refusals(call, lp_args, LOGITS + [
        (dict(lp=None), "RL_ERR_INVALID_ARG", "logprobs is NULL"),
        (dict(lp=fake([10], BF16)), "RL_ERR_DTYPE", "logprobs must be f32"),
        (dict(lp=fake([10], F32, strides=[0])), "RL_ERR_UNSUPPORTED", "logprobs"),
        (dict(ent=fake([9], F32)), "RL_ERR_SHAPE", "entropy"), (dict(lse=fake([11], F32)), "RL_ERR_SHAPE", "lse"),
        (dict(ids=None), "RL_ERR_INVALID_ARG", "must be given together"),
        (dict(lps=None), "RL_ERR_INVALID_ARG", "must be given together"),
        (dict(ids=fake([10, 3], I64)), "RL_ERR_DTYPE", "top_ids must be int32"),
        (dict(ids=fake([9, 3], I32)), "RL_ERR_SHAPE", "top_ids must be"),
        (dict(lps=fake([10, 4], F32)), "RL_ERR_SHAPE", "top_logprobs must be [10, 3]"),
        (dict(lps=fake([10, 3], F32, strides=[6, 2])), "RL_ERR_UNSUPPORTED", "top_logprobs"),
        (dict(ids=fake([10, 33], I32), lps=fake([10, 33], F32)), "RL_ERR_UNSUPPORTED", "at most 32"),
        (dict(x=fake([1 << 24, 100], BF16), tok=fake([1 << 24], I64)), "RL_ERR_UNSUPPORTED", "too large")])
    for name, make, needle in [
            ("lp", lambda a: fake([10], F32, a["x"].data + 1996), "logprobs and logits"),
            ("ent", lambda a: fake([10], F32, a["lp"].data + 4), "logprobs and entropy"),
            ("ids", lambda a: fake([10, 3], I32, a["ids"].data, [2, 1]), "top_ids: elements that are written"),
            ("ids", lambda a: fake([10, 3], I32, a["lps"].data), "top_ids and top_logprobs"),
            ("lse", lambda a: fake([10], F32, a["tok"].data + 76), "lse and tokens"),
            ("lps", lambda a: fake([10, 3], F32, a["scale"].data), "top_logprobs and row_scale")]:
        a = apart(lp_args())
        refused(call, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


def lp_grad_args(T=10, V=100, **kw):
    a = dict(x=fake([T, V], BF16), tok=fake([T], I64), scale=fake([T], F32), lse=fake([T], F32), ent=fake([T], F32),
             g=fake([T], F32), h=fake([T], F32), d=fake([T, V], BF16))
    return {**a, **kw}


def test_token_logprobs_backward_refuses():
    call = ra.lib().rl_attn_token_logprobs_backward
    refusals(call, lp_grad_args, LOGITS + [
        (dict(lse=None), "RL_ERR_INVALID_ARG", "lse is NULL"), (dict(ent=None), "RL_ERR_INVALID_ARG", "entropy is NULL"),
        (dict(g=None, h=None), "RL_ERR_INVALID_ARG", "both NULL"), (dict(g=fake([9], F32)), "RL_ERR_SHAPE", "d_logprobs"),
        (dict(h=fake([10], BF16)), "RL_ERR_DTYPE", "d_entropy"), (dict(d=None), "RL_ERR_INVALID_ARG", "d_logits is NULL"),
        (dict(d=fake([10, 100], F32)), "RL_ERR_DTYPE", "d_logits must be bf16"),
        (dict(d=fake([10, 101], BF16)), "RL_ERR_SHAPE", "d_logits must be [10, 100]"),
        (dict(d=fake([10, 100], BF16, strides=[99, 1])), "RL_ERR_UNSUPPORTED", "must not overlap"),
        (dict(x=fake([1 << 23, 5000], BF16), tok=fake([1 << 23], I64), scale=None, lse=fake([1 << 23], F32),
              ent=None, h=None, g=fake([1 << 23], F32), d=fake([1 << 23, 5000], BF16)), "RL_ERR_UNSUPPORTED",
         "too large")])
    for name, make, needle in [
            ("d", lambda a: fake([10, 100], BF16, a["x"].data + 2), "d_logits must be logits or not overlap it"),
            ("d", lambda a: fake([10, 100], BF16, a["x"].data, [101, 1]), "d_logits must be logits or not overlap it"),
            ("d", lambda a: fake([10, 100], BF16, a["lse"].data - 1998), "d_logits and lse"),
            ("g", lambda a: fake([10], F32, a["d"].data), "d_logits and d_logprobs")]:
        a = apart(lp_grad_args())
        refused(call, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


# --------------------------------------------------------------------------------- requests that begin and end

def fork_args(B=3, **kw):
    a = dict(par=fake([B], I32), n=fake([B], I32), kv=fake([B], I32), free=fake([20], I32), used=fake([1], I32),
             page=16, pages=30, table=fake([B, 4], I32), kv_out=fake([B], I32), used_out=fake([1], I32),
             copies=fake([B, 3], I32))
    return {**a, **kw}


TABLE = [
    (dict(kv=None), "RL_ERR_INVALID_ARG", "kv_lens is NULL"),
    (dict(kv=fake([3], I64)), "RL_ERR_DTYPE", "kv_lens must be int32"),
    (dict(free=None), "RL_ERR_INVALID_ARG", "free_pages is NULL"),
    (dict(free=fake([20], F32)), "RL_ERR_DTYPE", "free_pages"),
    (dict(used=fake([2], I32)), "RL_ERR_SHAPE", "free_used"),
    (dict(page=24), "RL_ERR_UNSUPPORTED", "page size"), (dict(page=256), "RL_ERR_UNSUPPORTED", "page size"),
    (dict(pages=-1), "RL_ERR_INVALID_ARG", "num_pages"), (dict(pages=1 << 31), "RL_ERR_UNSUPPORTED", "too large"),
    (dict(table=fake([2, 4], I32)), "RL_ERR_SHAPE", "block_table.shape[0]"),
    (dict(table=fake([3, 1 << 24], I32)), "RL_ERR_UNSUPPORTED", "too large"),
    (dict(kv_out=fake([3], I32, strides=[0])), "RL_ERR_UNSUPPORTED", "kv_lens_out: stride"),
    (dict(kv_out=None), "RL_ERR_INVALID_ARG", "kv_lens_out is NULL"),
    (dict(used_out=fake([1], I64)), "RL_ERR_DTYPE", "free_used_out"),
]


def test_fork_requests_refuses():
    call = ra.lib().rl_attn_fork_requests
    refusals(call, fork_args, TABLE + [
        (dict(par=fake([4], I32)), "RL_ERR_SHAPE", "parents must have 3"),
        (dict(n=fake([3], F32)), "RL_ERR_DTYPE", "fork_lens must be int32"),
        (dict(table=fake([3, 4], I32, strides=[0, 1])), "RL_ERR_UNSUPPORTED", "block_table"),
        (dict(copies=fake([3, 2], I32)), "RL_ERR_SHAPE", "copies must be [3, 3]"),
        (dict(copies=fake([3, 3], I32, strides=[1, 3])), "RL_ERR_UNSUPPORTED", "copies"),
        (dict(copies=fake([3, 3], I64)), "RL_ERR_DTYPE", "copies")])
    for name, make, needle in [
            ("kv_out", lambda a: fake([3], I32, a["kv"].data + 4), "kv_lens_out must be kv_lens"),
            ("kv_out", lambda a: fake([3], I32, a["par"].data), "kv_lens_out and parents"),
            ("copies", lambda a: fake([3, 3], I32, a["copies"].data, [2, 1]), "copies: elements that are written"),
            ("copies", lambda a: fake([3, 3], I32, a["table"].data + 44), "block_table and copies"),
            ("used_out", lambda a: fake([1], I32, a["free"].data + 8), "free_used_out and free_pages"),
            ("table", lambda a: fake([3, 4], I32, a["table"].data, [3, 1]), "block_table: elements that are written")]:
        a = apart(fork_args())
        refused(call, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


def test_copy_pages_refuses():
    def make(n=5, dtype=BF16, **kw):
        return {**dict(c=fake([n, 3], I32), k=fake([9, 16, 2, 128], dtype), v=fake([9, 16, 2, 128], dtype)), **kw}

    refusals(ra.lib().rl_attn_copy_pages, make, [
        (dict(c=None), "RL_ERR_INVALID_ARG", "copies is NULL"), (dict(c=fake([5, 2], I32)), "RL_ERR_SHAPE", "copies"),
        (dict(c=fake([5, 3], I64)), "RL_ERR_DTYPE", "copies"),
        (dict(c=fake([5, 3], I32, strides=[1, 5])), "RL_ERR_UNSUPPORTED", "copies"),
        (dict(k=None), "RL_ERR_INVALID_ARG", "k_pages is NULL"), (dict(dtype=F32), "RL_ERR_DTYPE", "k_pages"),
        (dict(v=fake([9, 16, 2, 128], FP8)), "RL_ERR_DTYPE", "v_pages must be bf16"),
        (dict(v=fake([8, 16, 2, 128], BF16)), "RL_ERR_SHAPE", "shapes differ"),
        (dict(k=fake([9, 16, 2, 64], BF16)), "RL_ERR_UNSUPPORTED", "head dimension"),
        (dict(k=fake([9, 24, 2, 128], BF16), v=fake([9, 24, 2, 128], BF16)), "RL_ERR_UNSUPPORTED", "page size"),
        (dict(dtype=FP8, k=fake([9, 16, 2, 128], FP8, strides=[4104, 256, 128, 1])), "RL_ERR_UNSUPPORTED", "16 bytes"),
        (dict(c=fake([1 << 23, 3], I32)), "RL_ERR_UNSUPPORTED", "copies too many")])


def test_drop_tokens_refuses():
    def make(B=3, **kw):
        a = dict(kv=fake([B], I32), keep=fake([B], I32), table=fake([B, 4], I32), page=16, pages=30,
                 free=fake([20], I32), used=fake([1], I32), kv_out=fake([B], I32), used_out=fake([1], I32))
        return {**a, **kw}

    call = ra.lib().rl_attn_drop_tokens
    refusals(call, make, TABLE + [
        (dict(keep=fake([4], I32)), "RL_ERR_SHAPE", "keep_lens must have 3"),
        (dict(keep=None), "RL_ERR_INVALID_ARG", "keep_lens is NULL"),
        (dict(free=fake([20], I32, strides=[0])), "RL_ERR_UNSUPPORTED", "free_pages: stride")])
    for name, change, needle in [
            ("free", lambda a: fake([20], I32, a["table"].data + 44), "free_pages and block_table"),
            ("free", lambda a: fake([20], I32, a["used"].data - 76), "free_pages and free_used"),
            ("kv_out", lambda a: fake([3], I32, a["keep"].data), "kv_lens_out and keep_lens"),
            ("kv_out", lambda a: fake([3], I32, a["kv"].data - 4), "kv_lens_out must be kv_lens"),
            ("used_out", lambda a: fake([1], I32, a["kv"].data), "free_used_out and kv_lens")]:
        a = apart(make())
        refused(call, {**a, name: change(a)}, "RL_ERR_UNSUPPORTED", needle)


def test_calls_without_rows_need_no_gpu():
    """Nothing to do, nothing launched."""
    n = norm_args(T=0)
    assert ra.lib().rl_attn_norm_rope(*(ctypes.byref(x) if isinstance(x, ra.RlTensor) else x for x in n.values()),
                                      None) == 0
    e = lp_args(T=0)
    assert ra.lib().rl_attn_token_logprobs(*(ctypes.byref(x) for x in e.values()), None) == 0
    g = lp_grad_args(T=0)
    assert ra.lib().rl_attn_token_logprobs_backward(*(ctypes.byref(x) for x in g.values()), None) == 0


def test_workspace_sizes_do_not_fall():
    size = ra.token_logprobs_workspace_size
    last = 0
    for rows in (1, 7, 100, 2047, 2048, 5000, 1 << 20):
        assert size(rows, 131072, 20) >= last and size(rows, 131072, 20) <= size(rows, 131073, 32)
        assert size(rows, 131072, 0) <= size(rows, 131072, 1)
        last = size(rows, 131072, 20)
    assert size(0, 10) == size(10, 0) == size(10, 10, 33) == size(10, 1 << 22) == 0
    assert ra.norm_rope_backward_workspace_size() > 0
