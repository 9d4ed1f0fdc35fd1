"""What the step's calls write may be what they read only as the same view, where that is said; the rest is refused before
anything is launched. Slices of one buffer that share no byte are taken."""

import numpy as np
import pytest
import torch

from paper_2609_08368_amd import rl_attn as ra
from tests.test_abi import FAKE, fake
from tests.test_step_abi import BF16, F32, FP8, I32, I64, append_args, map_args, prefill_args, refused, rope_args


def apart(args, **kw):
    """The tensors at addresses of their own."""
    for i, t in enumerate(args.values()):
        if isinstance(t, ra.RlTensor):
            t.data = FAKE + (i << 24)
    return {**args, **kw}


ROWS = 128 * 2                   # bytes of a head row


@pytest.mark.parametrize("name,make,needle", [
    ("kv_out", lambda a: fake([3], I32, a["new"].data), "kv_lens_out and new_lens"),
    ("kv_out", lambda a: fake([3], I32, a["new"].data + 8), "kv_lens_out and new_lens"),
    ("ptr", lambda a: fake([4], I32, a["new"].data - 12), "qo_indptr and new_lens"),
    ("ptr", lambda a: fake([4], I32, a["kv"].data), "qo_indptr and kv_lens"),
    ("pos", lambda a: fake([10], I32, a["slots"].data + 76), "slot_map and positions"),
    ("slots", lambda a: fake([10], I64, a["free"].data + 40), "slot_map and free_pages"),
    ("used_out", lambda a: fake([1], I32, a["kv"].data + 4), "free_used_out and kv_lens"),
    ("used_out", lambda a: fake([1], I32, a["free"].data + 76), "free_used_out and free_pages"),
    ("used_out", lambda a: fake([1], I32, a["ptr"].data + 12), "free_used_out and qo_indptr"),
    ("table", lambda a: fake([3, 4], I32, a["used"].data - 44), "block_table and free_used"),
    ("table", lambda a: fake([3, 4], I32, a["table"].data, [3, 1]), "block_table: elements that are written"),
    ("delta", lambda a: fake([3], I32, a["pos"].data + 4), "positions and pos_delta"),
    ("new", lambda a: fake([3], I32, a["table"].data + 12, [5]), "block_table and new_lens"),
])
def test_map_slots_refuses(name, make, needle):
    a = apart(map_args())
    refused(ra.lib().rl_attn_map_slots, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


ROPE = [
    ("q_out", lambda a: fake([10, 8, 128], BF16, a["q"].data + ROWS), "q_out must be q or not overlap it"),
    ("q_out", lambda a: fake([10, 8, 128], BF16, a["q"].data, [2048, 128, 1]), "q_out must be q or not overlap it"),
    ("q_out", lambda a: fake([10, 8, 128], BF16, a["k"].data + 19 * ROWS), "q_out and k"),
    ("k_out", lambda a: fake([10, 2, 128], BF16, a["k"].data - ROWS), "k_out must be k"),
    ("k_out", lambda a: fake([10, 2, 128], BF16, a["q"].data), "k_out and q"),
    ("k_out", lambda a: fake([10, 2, 128], BF16, a["q_out"].data + 79 * ROWS), "q_out and k_out"),
]


@pytest.mark.parametrize("name,make,needle", ROPE)
def test_rope_refuses(name, make, needle):
    a = apart(rope_args())
    refused(ra.lib().rl_attn_rope, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("name,make,needle", ROPE + [
    ("q_out", lambda a: fake([10, 8, 128], BF16, a["v"].data - 79 * ROWS), "q_out and v_new"),
    ("k_out", lambda a: fake([10, 2, 128], BF16, a["v"].data), "k_out and v_new")])
def test_rope_append_refuses(name, make, needle, fp8):
    a = apart(append_args(fp8), k_out=fake([10, 2, 128], BF16, FAKE + (1 << 30)))
    call = ra.lib().rl_attn_rope_append_kv_fp8 if fp8 else ra.lib().rl_attn_rope_append_kv
    refused(call, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


@pytest.mark.parametrize("name,make,needle", [
    ("out", lambda a: fake([10, 8, 128], BF16, a["k"].data), "out and k"),
    ("out", lambda a: fake([10, 8, 128], BF16, a["v"].data + 19 * ROWS), "out and v"),
    ("out", lambda a: fake([10, 8, 128], BF16, a["q"].data - ROWS), "out must be q"),
    ("out", lambda a: fake([10, 8, 128], F32, a["q"].data), "out must be q"),
    ("out", lambda a: fake([10, 8, 128], BF16, a["out"].data, [0, 128, 1]), "out: elements that are written"),
    ("out", lambda a: fake([10, 8, 128], BF16, a["out"].data, [1024, 64, 1]), "out: elements that are written"),
    ("lse", lambda a: fake([10, 8], F32, a["out"].data + 80 * ROWS - 4), "out and lse_out"),
    ("lse", lambda a: fake([10, 8], F32, a["k"].data), "lse_out and k"),
    ("lse", lambda a: fake([10, 8], F32, FAKE + (1 << 30), [8, 0]), "lse_out: elements that are written"),
])
def test_prefill_refuses(name, make, needle):
    a = apart(prefill_args())
    refused(ra.lib().rl_attn_prefill, {**a, name: make(a)}, "RL_ERR_UNSUPPORTED", needle)


DEV = "cuda:0"


@pytest.mark.gpu
def test_map_slots_takes_columns_of_one_buffer():
    kv, new = [20, 0, 7, 64], [1, 30, 0, 9]
    free = torch.arange(40, 60, dtype=torch.int32, device=DEV)
    table = torch.full((4, 9), -1, dtype=torch.int32, device=DEV)
    table[:, :5] = torch.arange(20, dtype=torch.int32, device=DEV).view(4, 5)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    want_table = table.clone()
    want = ra.map_slots(dev(kv), dev(new), free, dev([2]), want_table, 16, 64, 44, pos_delta=dev([0, -1, 5, 2]))
    # a request's lengths, its table and a row bound beside each other; lists as columns of another buffer
    one = torch.full((5, 14), -9, dtype=torch.int32, device=DEV)
    one[:4, 0], one[:4, 1], one[:4, 2], one[:4, 3:12], one[0, 13] = dev(kv), dev(new), dev([0, -1, 5, 2]), table, 2
    rows = torch.zeros((44, 2), dtype=torch.int64, device=DEV)
    used = one[:1, 13]
    m = ra.map_slots(one[:4, 0], one[:4, 1], free, used, one[:4, 3:12], 16, 64, pos_delta=one[:4, 2],
                     kv_lens_out=one[:4, 0], free_used_out=used, qo_indptr=one[:, 12], slot_map=rows[:, 0],
                     positions=rows.view(torch.int32)[:, 2])
    ra.check_device_errors()
    for x, y in zip(m, want):
        assert torch.equal(x, y)
    assert torch.equal(one[:4, 3:12], want_table) and torch.all(one[4, :12] == -9)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_rope_append_in_place_in_a_fused_buffer(fp8):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    qkv = torch.randn(50, 12, 128, generator=g, device=DEV).to(torch.bfloat16)
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    pools = [torch.zeros(9, 8, 2, 128, device=DEV).to(kind) for _ in range(4)]
    scales = [torch.tensor([0.02, 0.03], device=DEV)] * 2 if fp8 else []
    pos, slots = torch.arange(50, dtype=torch.int32, device=DEV)[None], torch.randperm(72, generator=g, device=DEV)[:50]
    freq = torch.tensor(1e4 ** (-np.arange(64) / 64), dtype=torch.float32, device=DEV)
    call = ra.rope_append_kv_fp8 if fp8 else ra.rope_append_kv
    k = torch.empty(50, 2, 128, dtype=torch.bfloat16, device=DEV)
    q = call(qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], pos, freq, slots, *pools[:2], *scales, k_out=k)
    mine = qkv.clone()
    call(mine[:, :8], mine[:, 8:10], mine[:, 10:], pos, freq, slots, *pools[2:], *scales, q_out=mine[:, :8],
         k_out=mine[:, 8:10])
    ra.check_device_errors()
    assert torch.equal(mine, torch.cat((q, k, qkv[:, 10:]), dim=1))
    for a, b in zip(pools[:2], pools[2:]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # query and key rows alternating head by head, as the outputs are
    turns = torch.stack((qkv[:, :6], qkv[:, 6:]), dim=2).reshape(50, 12, 128).contiguous()
    out = turns.clone()
    q, k = ra.rope(turns[:, 0::2], turns[:, 1::2], pos, freq)
    ra.rope(out[:, 0::2], out[:, 1::2], pos, freq, q_out=out[:, 0::2], k_out=out[:, 1::2])
    assert torch.equal(out[:, 0::2], q) and torch.equal(out[:, 1::2], k)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv", [(8, 2), (32, 32), (96, 8), (300, 1)])
def test_prefill_in_place(hq, hkv):
    """The output over the query rows of a fused projection; with scores that make a wave compute its rows twice."""
    lens = [130, 0, 700, 33, 1, 257]
    g = torch.Generator(device=DEV)
    g.manual_seed(hq)
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)
    qkv = torch.randn(sum(lens), hq + 2 * hkv, 128, generator=g, device=DEV).to(torch.bfloat16)
    qkv[130 + 400:130 + 420, hq:hq + hkv] *= 60.0
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    lse, lse2 = (torch.zeros(qkv.shape[0], hq, device=DEV) for _ in range(2))
    want = ra.prefill(q, k, v, ptr, 128 ** -0.5, lse=lse)
    kv = qkv[:, hq:].clone()
    assert ra.prefill(q, k, v, ptr, 128 ** -0.5, out=q, lse=lse2) is q
    ra.check_device_errors()
    assert torch.isfinite(want).all() and torch.equal(q, want) and torch.equal(lse, lse2)
    assert torch.equal(qkv[:, hq:], kv)
