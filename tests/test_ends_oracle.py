"""The definitions of the operators at a step's ends against differences and against what they have to keep (CPU)."""

import numpy as np
import pytest

from oracle import ends


def differences(f, x, d, step=1e-6):
    """Directional derivative of f at x along d, by central differences."""
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("freqs", [8, 40, 64])
def test_norm_rope_gradient_is_the_difference(freqs, interleaved):
    """Steps of 1e-6 leave 1e-12 of the third derivative and 1e-16 / 1e-6 of rounding: 1e-8 of the sum of magnitudes."""
    rng = np.random.default_rng(freqs)
    x, dy, w = rng.standard_normal((3, 2, 128)), rng.standard_normal((3, 2, 128)), rng.uniform(0.5, 2, 128)
    args = (1e-6, rng.integers(0, 5000, (2, 3)), 1e4 ** (-np.arange(freqs) / freqs), np.arange(freqs) % 2, interleaved)
    dx, dw = ends.norm_rope_backward(dy, x, w, *args)
    for _ in range(4):
        d = rng.standard_normal(x.shape)
        want = differences(lambda v: (ends.norm_rope(v, w, *args) * dy).sum(), x, d)
        assert abs((dx * d).sum() - want) <= 1e-8 * np.abs(dx * d).sum() + 1e-8
        d = rng.standard_normal(128)
        want = differences(lambda v: (ends.norm_rope(x, v, *args) * dy).sum(), w, d)
        assert abs((dw * d).sum() - want) <= 1e-8 * np.abs(dw * d).sum() + 1e-8


def test_logprobs_gradient_is_the_difference():
    rng = np.random.default_rng(1)
    x, g, h = 3 * rng.standard_normal((5, 37)), rng.standard_normal(5), rng.standard_normal(5)
    tokens, scale = np.array([3, 36, -1, 0, 7]), rng.uniform(0.5, 2, 5).astype(np.float32)

    def loss(v):
        f = ends.token_logprobs(v, tokens, scale)
        return (f["logprobs"] * g + f["entropy"] * h).sum()

    d_x = ends.token_logprobs_backward(x, tokens, g, h, scale)
    assert np.all(d_x[2] == 0) and np.abs(d_x.sum(-1)).max() < 1e-12, "a constant added to a row changes nothing"
    for _ in range(5):
        d = rng.standard_normal(x.shape)
        assert abs((d_x * d).sum() - differences(loss, x, d)) <= 1e-8 * np.abs(d_x * d).sum() + 1e-8


def test_logprobs_of_rows_that_exclude_tokens():
    x = np.array([[1.0, -np.inf, 2.0, 2.0], [-np.inf] * 4, [0.0, np.nan, np.inf, 1.0], [5.0, 5.0, 5.0, 5.0]])
    f = ends.token_logprobs(x, [1, 0, 3, 3], top=3)
    assert f["logprobs"][0] == -np.inf and f["logprobs"][1] == -np.inf and np.isnan(f["logprobs"][2])
    assert f["entropy"][1] == 0 and np.isclose(f["entropy"][3], np.log(4)) and f["lse"][1] == -np.inf
    assert f["top_ids"].tolist() == [[2, 3, 0], [-1, -1, -1], [2, 3, 0], [0, 1, 2]]
    d = ends.token_logprobs_backward(x[:2], [1, 0], np.ones(2), np.ones(2))
    assert np.isfinite(d).all() and d[0, 1] == 1.0 and np.all(d[1] == 0)


def lively(seed, batch=40, page=16, pool=900):
    """Steps of a pool's life: requests grow from the list, fork and drop; what the tables and the list say."""
    rng = np.random.default_rng(seed)
    lens, table = np.zeros(batch, np.int64), np.full((batch, 12), -1)
    free, used = rng.permutation(pool), 0
    for _ in range(60):
        new = np.where(rng.random(batch) < 0.5, rng.integers(0, 40, batch), 0)
        for b in range(batch):                             # growth, as a slot map places it
            # only into pages of its own
            n = min(int(new[b]), 12 * page - int(lens[b]))
            while n and -(-(lens[b] + n) // page) - -(-lens[b] // page) > len(free) - used:
                n -= 1
            for j in range(-(-lens[b] // page), -(-(lens[b] + n) // page)):
                table[b, j] = free[used]
                used += 1
            lens[b] += n
        yield lens, table, free, used
        keep = np.where(rng.random(batch) < 0.3, 0, np.where(rng.random(batch) < 0.2, lens // page * page, lens))
        d = ends.drop_tokens(lens, keep, table, free, used, page, pool)
        assert not d["errors"]
        lens, free, used = d["kv_lens"], d["free_pages"], d["free_used"]
        yield lens, table, free, used
        parents = np.full(batch, -1)
        for b in np.flatnonzero(lens == 0):
            p = int(rng.integers(batch))
            if lens[p] > 0:
                parents[b] = p
        f = ends.fork_requests(parents, np.where(parents < 0, 0, lens[parents] * rng.random(batch)), lens, free, used,
                               table, page, pool)
        assert not f["errors"]
        lens, table, used = f["kv_lens"], f["block_table"], f["free_used"]


@pytest.mark.parametrize("seed", range(3))
def test_every_page_is_held_or_listed_once(seed):
    for lens, table, free, used in lively(seed):
        held = {int(p) for b, n in enumerate(lens) for p in table[b, :-(-n // 16)]}
        listed = [int(p) for p in free[used:]]
        assert len(set(listed)) == len(listed) and not held & set(listed) and len(held) + len(listed) == 900
        # a partly filled page has one holder
        last = [int(table[b, n // 16]) for b, n in enumerate(lens) if n % 16]
        whole = {int(p) for b, n in enumerate(lens) for p in table[b, :n // 16]}
        assert len(set(last)) == len(last) and not whole & set(last)
