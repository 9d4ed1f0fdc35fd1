"""A request that is cut back inside a page it shares goes on as another one: forked there, copied, ended. What it writes next
is its own, and the pages of the others stay as they are."""

import numpy as np
import pytest
import torch

from oracle import ends
from paper_2609_08368_amd import rl_attn as ra
from tests.test_gpu_step import dev, rand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("keep", [1, 16, 20, 31, 32])
def test_cut_inside_a_shared_page(keep):
    P, layers, pool = 16, 2, 12
    table = dev(np.array([[7, 3, 9, -1, -1], [7, 3, 2, -1, -1], [7, 3, 5, -1, -1], [-1] * 5]))
    lens, used = dev(np.array([40, 37, 33, 0])), dev(np.array([6]))
    free = dev(np.array([7, 3, 9, 2, 5, 0, 11, 10, 8, 6, 4, 1]))          # (six are taken)
    pages = [[rand(8 * i + j, pool, P, 2, 128) for j in range(2)] for i in range(layers)]
    before = [[x.clone() for x in layer] for layer in pages]
    f = ra.fork_requests(dev(np.array([-1, -1, -1, 1])), dev(np.array([0, 0, 0, keep])), lens, free, used, table, P, pool,
                         kv_lens_out=lens, free_used_out=used)
    for k, v in pages:
        ra.copy_pages(f.copies, k, v)
    want = ends.drop_tokens([40, 37, 33, keep], [99, 0, 99, 99], table.cpu().numpy(), free.cpu().numpy(), int(used), P, pool)
    ra.drop_tokens(lens, dev(np.array([99, 0, 99, 99])), table, free, used, P, pool, kv_lens_out=lens, free_used_out=used)
    assert lens.tolist() == [40, 0, 33, keep] == list(want["kv_lens"]) and free.tolist() == list(want["free_pages"])
    assert 2 in free[int(used):].tolist() and not {3, 7} & set(free[int(used):].tolist())
    # three turns' rows behind what it kept, as many as fill the page and begin others
    rows = torch.cat([rand(90 + i, n, 2, 128) for i, n in enumerate((1, 16, 20))])
    at = 0
    for n in (1, 16, 20):
        m = ra.map_slots(lens, dev(np.array([0, 0, 0, n])), free, used, table, P, pool, n, kv_lens_out=lens,
                         free_used_out=used)
        for k, v in pages:
            k.view(-1, 2, 128)[m.slot_map] = rows[at:at + n]
            v.view(-1, 2, 128)[m.slot_map] = rows[at:at + n]
        at += n
    ra.check_device_errors()
    now = table.cpu().numpy()
    for layer, old in zip(pages, before):
        for x, y in zip(layer, old):
            for page in (7, 3, 9, 5):                                     # of the others
                assert torch.equal(x[page], y[page])
            mine = x[dev(now[3, :-(-(keep + 37) // P)], torch.int64)].reshape(-1, 2, 128)[:keep + 37]
            prompt = y[dev(np.array([7, 3]), torch.int64)].reshape(-1, 2, 128)[:keep]
            assert torch.equal(mine, torch.cat((prompt, rows)))
