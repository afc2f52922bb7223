"""libra_kv_accept over batches of many requests: every request's tokens move, those of the last too."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra

from test_gpu_kv_append import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,hkv", [(1 << 21, 9), ((1 << 24) + 5, 1)])
def test_more_workgroups_than_a_launch_takes(batch, hkv):
    """Requests that share a page and accept nothing, and among them some of a page each that accept node 3."""
    cache = Cache(12, hkv)
    movers = np.array([0, 1, batch // 2, batch // 8 * 7, batch - 2, batch - 1])
    counts = torch.zeros(batch, dtype=torch.int32, device="cuda")
    table = torch.full((batch, 1), 11, dtype=torch.int32, device="cuda")
    prior = torch.full((batch,), 4, dtype=torch.int32, device="cuda")
    accepted = torch.full((batch, 1), 3, dtype=torch.int32, device="cuda")
    at = torch.from_numpy(movers).cuda()
    counts[at] = 1
    table[at, 0] = torch.arange(len(movers), dtype=torch.int32, device="cuda")
    libra.libra_kv_accept(cache.layout, prior, accepted, counts, table, 1)
    got, want = cache.logical(), cache.initial()
    for g, w in zip(got, want):
        for page in range(len(movers)):
            w[page * 16 + 4] = w[page * 16 + 7]
        assert torch.equal(g.view(torch.int16), w.view(torch.int16))
    cache.close()
