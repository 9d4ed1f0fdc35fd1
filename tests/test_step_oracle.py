"""The plain definitions of a step (slot maps, rotary positions, whole prompts) against what mathematics fixes (CPU)."""

import numpy as np
import pytest
import torch

import oracle
from oracle import step


def _lens(rng, n, page):
    cached = rng.integers(0, 5 * page, n)
    return cached, rng.integers(0, 3 * page, n)


@pytest.mark.parametrize("page", [8, 64])
def test_map_gives_every_new_token_a_place_of_its_own(page):
    rng = np.random.default_rng(page)
    cached, new = _lens(rng, 9, page)
    before = -(-cached // page)
    ids = rng.permutation(200)
    table = np.full((9, 12), -7)
    at = 0
    for b, p in enumerate(before):
        table[b, :p] = ids[at:at + p]
        at += p
    free = ids[at:]
    m = step.map_slots(cached, new, free, 3, table, page, 200, int(new.sum()) + 5, pos_delta=np.arange(9) - 4)
    assert not m["errors"] and np.array_equal(m["kv_lens"], cached + new)
    used = (-(-(cached + new) // page) - before).sum()
    assert m["free_used"] == 3 + used
    # every token of every request has a slot that no other has, and the table agrees with the slot map
    seen = set()
    for b in range(9):
        for t in range(int(m["kv_lens"][b])):
            s = int(m["block_table"][b, t // page]) * page + t % page
            assert s not in seen
            seen.add(s)
            if t >= cached[b]:
                r = m["qo_indptr"][b] + t - cached[b]
                assert m["slot_map"][r] == s and m["positions"][r] == t + b - 4
        assert np.all(m["block_table"][b, -(-int(m["kv_lens"][b]) // page):] == -7)
    assert np.all(m["slot_map"][-5:] == -1) and np.all(m["positions"][-5:] == 0)


def test_map_refuses_a_request_that_is_longer_than_its_table():
    table = np.zeros((4, 2), int)
    one = dict(free_pages=[5, 6, 7], free_used=0, block_table=table, page_size=8, num_pages=8)
    m = step.map_slots([0, 0, 0, -1], [8, 17, 9, 1], rows=99, **one)
    assert m["errors"] == {"length-out-of-range"} and m["qo_indptr"].tolist() == [0, 8, 8, 17, 17]
    assert m["free_used"] == 3 and m["kv_lens"].tolist() == [8, 0, 9, -1]
    assert m["block_table"].tolist() == [[5, 0], [0, 0], [6, 7], [0, 0]]


def test_map_stops_at_the_first_that_does_not_fit():
    table = np.zeros((3, 2), int)
    one = dict(free_pages=[5, 6, 7], free_used=1, block_table=table, page_size=8, num_pages=8)
    m = step.map_slots([0, 0, 0], [8, 9, 1], rows=99, **one)
    assert m["errors"] == {"free-pages-exhausted"} and m["qo_indptr"].tolist() == [0, 8, 8, 8]
    assert m["free_used"] == 2 and m["kv_lens"].tolist() == [8, 0, 0]
    m = step.map_slots([0, 0, 0], [1, 8, 1], rows=5, **one)
    assert m["errors"] == {"rows-past-slot-map"} and m["qo_indptr"].tolist() == [0, 1, 1, 1]


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_keeps_lengths_and_sees_differences_only(interleaved):
    rng = np.random.default_rng(3)
    f = 10000.0 ** (-np.arange(24) / 24)
    axes = np.arange(24) % 3
    q, k = rng.standard_normal((2, 5, 3, 128))
    p, s = rng.integers(-50, 5000, (3, 5)), rng.integers(-50, 5000, (3, 5))
    qr, kr = step.rope(q, p, f, axes, interleaved), step.rope(k, s, f, axes, interleaved)
    assert np.allclose(np.linalg.norm(qr, axis=-1), np.linalg.norm(q, axis=-1))
    assert np.array_equal(qr[..., 48:], q[..., 48:])
    back = step.rope(qr, p, f, axes, interleaved, inverse=True)
    assert np.allclose(back, q, atol=1e-12)
    # q(p) . k(s) = q(p - s) . k(0)
    rel = step.rope(q, p - s, f, axes, interleaved)
    assert np.allclose((qr * kr).sum(-1), (rel * k).sum(-1), atol=1e-11)
    # the gradient is the rotation back
    x = torch.tensor(q, requires_grad=True)
    lo, hi = (slice(0, 48, 2), slice(1, 48, 2)) if interleaved else (slice(0, 24), slice(24, 48))
    a = torch.tensor(p.astype(np.float64)[axes].T * f.astype(np.float32))[:, None]
    y = (x[..., lo] * a.cos() - x[..., hi] * a.sin()) * torch.tensor(kr[..., lo])
    y = y + (x[..., hi] * a.cos() + x[..., lo] * a.sin()) * torch.tensor(kr[..., hi])
    (y.sum() + (x[..., 48:] * torch.tensor(kr[..., 48:])).sum()).backward()
    assert np.allclose(x.grad.numpy(), step.rope(kr, p, f, axes, interleaved, inverse=True), atol=1e-9)


def test_rope_of_position_one_by_hand():
    x = np.zeros((1, 1, 128))
    x[0, 0, 3] = 2.0
    half = step.rope(x, [[1]], [0.1 * i for i in range(8)])
    assert np.isclose(half[0, 0, 3], 2 * np.cos(np.float32(0.3)), atol=1e-7)
    assert np.isclose(half[0, 0, 11], 2 * np.sin(np.float32(0.3)), atol=1e-7)
    pair = step.rope(x, [[1]], [0.1 * i for i in range(8)], interleaved=True)     # dimension 3 pairs with 2, frequency 1
    assert np.isclose(pair[0, 0, 3], 2 * np.cos(np.float32(0.1)), atol=1e-7)
    assert np.isclose(pair[0, 0, 2], -2 * np.sin(np.float32(0.1)), atol=1e-7)


def test_prefill_is_extend_from_an_empty_cache():
    rng = np.random.default_rng(5)
    lens = [5, 0, 17, 1]
    indptr = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = (rng.standard_normal((int(indptr[-1]) + 2, h, 16)) for h in (6, 2, 2))
    out, lse, spread = step.prefill(q, k, v, indptr, 0.25)
    pages_k, pages_v = np.zeros((len(lens) * 3, 8, 2, 16)), np.zeros((len(lens) * 3, 8, 2, 16))
    table = np.arange(len(lens) * 3).reshape(len(lens), 3)
    for b, n in enumerate(lens):
        for t in range(n):
            pages_k[table[b, t // 8], t % 8] = k[indptr[b] + t]
            pages_v[table[b, t // 8], t % 8] = v[indptr[b] + t]
    o, l = oracle.extend(q[:indptr[-1]], indptr, pages_k, pages_v, table, lens, 0.25)
    assert np.allclose(out[:indptr[-1]], o) and np.allclose(lse[:indptr[-1]], l)
    assert np.all(out[indptr[-1]:] == 0) and np.all(spread + 1e-12 >= np.abs(out))
