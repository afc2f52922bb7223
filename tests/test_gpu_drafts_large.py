"""The drafted step's operators at sizes that take several launches, or offsets past 32 bits: the bits of the
same work at small ones."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra

from test_gpu_kv_append import randn
from test_gpu_norm_rotary import EPS, Handle, run_backward, run_forward, weights
from test_gpu_tree import I32, SCALE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,rdim,hq,hk", [(8, 8, 1, 1), (6, 4, 2, 1), (8, 8, 0, 1)])
def test_norms_of_many_rows(dim, rdim, hq, hk):
    """More rows than one launch takes (2^24 heads), the gradients' sums within their rounding."""
    hd, rows = Handle(dim, rdim), 2 ** 24 // (hq + hk) + 301
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((rows, hq + hk, dim), device="cuda", generator=g).bfloat16()
    q, k = (x[:, :hq] if hq else None), x[:, hq:]
    wq, wk = weights(dim, torch.float32, 2) if hq else None, weights(dim, torch.float32, 3)
    pos = np.arange(rows) % 5000
    qo, ko = run_forward(hd, q, k, wq, wk, pos)
    at = np.concatenate([np.arange(40), np.arange(2 ** 24 // (hq + hk) - 40, rows)])
    t = torch.from_numpy(at).cuda()
    few = run_forward(hd, q[t] if hq else None, k[t], wq, wk, pos[at])
    assert torch.equal(ko[t], few[1]) and (not hq or torch.equal(qo[t], few[0]))
    assert ko.isfinite().all()
    _, dk, _, dw = run_backward(hd, None, k, None, wk, pos, None, ko)
    _, few_dk, _, _ = run_backward(hd, None, k[t], None, wk, pos[at], None, ko[t])
    assert torch.equal(dk[t], few_dk) and dw.isfinite().all()


def test_caches_past_4_gib():
    """K and V of 9.8 GB each: pages at both ends of it, against a cache of these pages alone."""
    pool, hkv, hq, few = 300_000, 8, 16, 60
    rng = np.random.default_rng(5)
    rot = libra.libra_rotary_create(base=1e6)
    wq, wk = (1 + 0.2 * torch.randn((2, 128), device="cuda")).bfloat16()
    prior, nodes = np.array([333, 40, 500]), np.array([9, 1, 30])
    B, rows = 3, int(nodes.sum())
    pages = -(-(prior + nodes) // 16)
    far = np.concatenate([np.arange(few // 2), np.arange(pool - few // 2, pool)])   # of page i of the small cache
    order, at = rng.permutation(few)[:pages.sum()], np.concatenate([[0], np.cumsum(pages)])
    k0, v0 = (randn((few, hkv, 16, 128), torch.bfloat16, s) for s in (1, 2))
    qkv = randn((rows, hq + 2 * hkv, 128), torch.bfloat16, 3)
    q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    starts = np.concatenate([[0], np.cumsum(nodes)])
    accepted, counts = np.array([[0, 3, 8], [0, 0, 0], [4, 11, 29]]), np.array([3, 1, 3])
    dev = lambda a, t=I32: torch.as_tensor(np.asarray(a), dtype=t).cuda()
    results = []
    for where in (np.arange(few), far):
        n = int(where.max()) + 1
        kc, vc = (torch.empty(n * hkv * 2048, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        lay = libra.libra_kv_layout_create(kc, vc, n, hkv)
        half = few // 2
        for first, part in ((int(where[0]), slice(0, half)), (int(where[half]), slice(half, few))):
            libra.libra_kv_pack_pages(lay, k0[part].contiguous(), v0[part].contiguous(), first, half)
        table, slots, positions = np.zeros((B, pages.max()), int), [], []
        for b in range(B):
            table[b, :pages[b]] = where[order[at[b]:at[b + 1]]]
            t = prior[b] + np.arange(nodes[b])
            slots += list(table[b, t // 16] * 16 + t % 16)
            positions += list(t)
        q_out, out = (torch.zeros((rows, hq, 128), dtype=torch.bfloat16, device="cuda") for _ in "qo")
        libra.libra_kv_append_norm(lay, rot, dev(positions), dev(slots, torch.int64), q, k, v, wq, wk, EPS, q_out)
        ws = torch.zeros(libra.libra_tree_attn_workspace_bytes(rows, B, hq, hkv), dtype=torch.uint8, device="cuda")
        libra.libra_tree_attn(lay, q_out, dev(prior), dev(starts), None, dev(table), table.shape[1], hq, SCALE, ws, out)
        libra.libra_kv_accept(lay, dev(prior), dev(accepted), dev(counts), dev(table), table.shape[1])
        got = []
        for first in (int(where[0]), int(where[half])):
            a, b = (torch.empty((half, hkv, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv")
            libra.libra_kv_unpack_pages(lay, a, b, first, half)
            got += [a, b]
        torch.cuda.synchronize()
        results.append([x.view(torch.int16) for x in (q_out, out, *got)])
        libra.libra_kv_layout_destroy(lay)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert results[0][1].any()
    libra.libra_rotary_destroy(rot)
