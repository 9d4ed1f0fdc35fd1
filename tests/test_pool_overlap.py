"""Page copies refuse pools whose rows overlap, and calls that append refuse rows that are written into the pages they write,
before anything is launched; slices of one buffer that share no byte are taken, and copied right."""

import numpy as np
import pytest
import torch

from paper_2609_08368_amd import rl_attn as ra
from tests.test_abi import FAKE, fake
from tests.test_ends_abi import EPS, refusals
from tests.test_step_abi import BF16, FP8, I32, append_args, refused

ROWS = 128 * 2                   # bytes of a head row
POOL = 9 * 16 * 2 * ROWS         # of a dense pool
SHAPE = [9, 16, 2, 128]


def copy_args(**kw):
    return {**dict(c=fake([5, 3], I32, FAKE + (1 << 30)), k=fake(SHAPE, BF16), v=fake(SHAPE, BF16, FAKE + (1 << 24))), **kw}


def test_copy_pages_refuses_overlaps():
    at = lambda ptr, strides=None, dtype=BF16: fake(SHAPE, dtype, ptr, strides)
    k = "k_pages: elements that are written"
    apart = "k_pages must be v_pages or not overlap it"
    refusals(ra.lib().rl_attn_copy_pages, copy_args, [(change, "RL_ERR_UNSUPPORTED", needle) for change, needle in [
        (dict(k=at(FAKE, [0, 256, 128, 1])), k),                       # one page for all
        (dict(k=at(FAKE, [4096, 0, 128, 1])), k),                      # one slot
        (dict(k=at(FAKE, [4096, 256, 0, 1])), k),                      # one head
        (dict(k=at(FAKE, [4096, 256, 64, 1])), k),                     # half a head
        (dict(k=at(FAKE, [4088, 256, 128, 1])), k),
        (dict(k=at(FAKE, [8192, 136, 2160, 1])), k),                   # the last slot of a head and the first of the next
        (dict(v=at(FAKE + (1 << 24), [4096, 128, 128, 1])), "v_pages: elements that are written"),
        (dict(v=at(FAKE + ROWS)), apart), (dict(v=at(FAKE + POOL - 16)), apart), (dict(v=at(FAKE - POOL + 16)), apart),
        (dict(k=at(FAKE, [8192, 256, 128, 1]), v=at(FAKE + 8192 - 16, [8192, 256, 128, 1])), apart),
        (dict(k=at(FAKE, [4096, 128, 2048, 1]), v=at(FAKE, [4096, 256, 128, 1])), apart),
        (dict(k=at(FAKE, [16384, 640, 256, 1]), v=at(FAKE + 2 * 640 + 16, [16384, 640, 256, 1])), apart),
        (dict(c=fake([5, 3], I32, FAKE + POOL - 4)), "k_pages and copies"),
        (dict(c=fake([5, 3], I32, FAKE - 56)), "k_pages and copies"),
        (dict(c=fake([5, 3], I32, FAKE + (1 << 24) + 32)), "v_pages and copies"),
        (dict(k=at(FAKE, dtype=FP8), v=at(FAKE + POOL // 2 - 16, dtype=FP8)), apart)]])


def test_copy_of_nothing_in_pools_of_no_pages():
    none = lambda *shape: fake(list(shape), BF16)
    call = lambda **kw: ra.lib().rl_attn_copy_pages(*(ra.ctypes.byref(t) for t in copy_args(**kw).values()), None)
    assert call(c=fake([0, 3], I32), v=fake(SHAPE, BF16)) == 0
    assert call(k=none(9, 16, 0, 128), v=none(9, 16, 0, 128)) == 0


@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
def test_append_refuses_rows_in_the_pages(fp8, normed):
    a = append_args(fp8)
    if normed:
        names = list(a)
        at = names.index("v") + 1
        w = dict(qw=fake([128], BF16), kw=fake([128], BF16), eps=EPS)
        a = {k: {**a, **w}[k] for k in names[:at] + list(w) + names[at:]}
    a["k_out"] = fake([10, 2, 128], BF16)
    for i, name in enumerate(a):
        if isinstance(a[name], ra.RlTensor):             # addresses of their own
            a[name] = fake(list(a[name].shape[:a[name].ndim]), a[name].dtype, FAKE + (i << 24))
    call = getattr(ra.lib(), f"rl_attn_{'norm_' * normed}rope_append_kv{'_fp8' * fp8}")
    pool = int(np.prod(a["kp"].shape[:4])) * (1 if fp8 else 2)
    for name, heads in (("q_out", 8), ("k_out", 2)):
        for pages in ("kp", "vp"):
            for at in (0, pool - 16, 16 - 10 * heads * ROWS):
                refused(call, {**a, name: fake([10, heads, 128], BF16, a[pages].data + at)}, "RL_ERR_UNSUPPORTED",
                        f"{name} and {pages[0]}_pages must not overlap")


def pieces(offset, shape, strides):
    """Of 16 bytes each, those of every head row."""
    n = [np.arange(s) * t // 8 for s, t in zip(shape, strides)]
    at = offset // 8 + n[0][:, None, None, None] + n[1][:, None, None] + n[2][:, None] + np.arange(16)
    return at.ravel()


@pytest.mark.gpu
def test_copies_take_slices_that_share_no_byte():
    """Pools of any order, padded, interleaved, one in the gaps of the other: refused if and only if they share a byte (two
    pools with the same strides), and copied as pools of their own are."""
    dev, rng, taken, refused = "cuda:0", np.random.default_rng(3), 0, 0
    data = torch.arange(1 << 15, dtype=torch.int32, device=dev).view(torch.bfloat16)
    copies = torch.tensor([[0, 1, 5]], dtype=torch.int32, device=dev)
    for turn in range(600):
        shape = (2 + int(rng.integers(2)), 8, int(rng.integers(1, 4)))
        order, strides, step = rng.permutation(3), [0, 0, 0], 128
        for i in order:                                  # dense or padded, now and then too narrow
            strides[i] = step + int(rng.choice([0, 0, 0, 8, 128, 256, 128 * int(rng.integers(1, 9)), -8]))
            step = max(128, strides[i] * shape[i])
        if turn % 7 == 0:
            strides[int(rng.integers(3))] = int(rng.integers(0, 30)) * 8
        same = turn % 5 != 0
        other = strides if same else [s + 8 * int(rng.integers(2)) for s in strides]
        extent = lambda st: sum((n - 1) * s for n, s in zip(shape, st)) + 128
        most = data.numel() - max(extent(strides), extent(other))
        if most < 8:
            continue
        a = int(rng.integers(most // 8)) * 8
        near = [0, 8, 128, -128, 256, 128 * shape[2], 128 * 8, 128 * 8 * shape[2], extent(strides), -extent(other)]
        b = int(np.clip(a + int(rng.choice(near)) * int(rng.choice([1, 1, 2])), 0, most // 8 * 8))
        pa, pb = pieces(a, shape, strides), pieces(b, shape, other)
        own = len(set(pa)) < len(pa) or len(set(pb)) < len(pb)
        one = a == b and all(n == 1 or s == t for n, s, t in zip(shape, strides, other))
        shared = not one and bool(set(pa) & set(pb))
        buffer = data.clone()
        k, v = (torch.as_strided(buffer, shape + (128,), tuple(st) + (1,), at) for st, at in ((strides, a), (other, b)))
        want = [x.clone() for x in (k, v)]
        try:
            ra.copy_pages(copies, k, v)
        except ra.RlAttnError as e:
            assert e.status == "RL_ERR_UNSUPPORTED"
            # (of other strides, by their ranges)
            meet = a < b + extent(other) and b < a + extent(strides)
            assert own or shared or (not same and meet), (shape, strides, other, a, b)
            refused += 1
            continue
        assert not own and not shared, (shape, strides, other, a, b)
        for x in want:
            x[1, :5] = x[0, :5]
        assert torch.equal(k.view(torch.int16), want[0].view(torch.int16)), (shape, strides, other, a, b)
        assert torch.equal(v.view(torch.int16), want[1].view(torch.int16))
        taken += 1
    ra.check_device_errors()
    assert taken > 150 and refused > 100, (taken, refused)
