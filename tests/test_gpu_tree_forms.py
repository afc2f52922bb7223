"""Tree attention where its forms meet, over long ranges, and captured with the calls around it.

The kernel takes four waves (tiles of 128 rows) where the mean request has 65 to 128 rows a KV head, eight (256
rows) otherwise, and counts an item's fixed cost differently above 128.  Tolerances: as in test_gpu_tree.py and
tree_codes.py."""
import numpy as np
import pytest
import torch

import tree_codes
from paper_2606_03077_amd import libra

from test_gpu_kv_append import Cache
from test_gpu_tree import I32, SCALE, Step, f64, run, tree_masks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["tree", "chain"])
@pytest.mark.parametrize("nodes", [63, 64, 65, 127, 128, 129, 255, 256])
@pytest.mark.parametrize("prior", [(0, 31, 700), (2500, 5, 64)])
def test_rows_on_both_sides_of_the_forms(nodes, prior, kind):
    """One query head to a KV head, so that as many rows as nodes."""
    run(prior, [nodes] * 3, 2, 2, kind, padding=0)


@pytest.mark.parametrize("group,most", [(8, 24), (7, 32), (8, 32), (8, 40), (16, 15), (3, 85), (2, 128)])
def test_uneven_trees_whose_mean_takes_four_waves(group, most):
    """Trees of up to more rows than a tile of 128, which are cut there, beside small ones."""
    rng = np.random.default_rng(group * most)
    nodes = rng.integers(1, most, size=24, endpoint=True)
    mean = lambda: -(-int(nodes.sum()) // 24) * group
    nodes[5] = most
    while mean() > 128:
        nodes = np.maximum(nodes - 1, 1)
        nodes[5] = most
    assert 64 < mean() <= 128
    run(rng.integers(0, 900, size=24).tolist(), nodes.tolist(), 2 * group, 2, padding=0)


def test_one_long_context_among_short_ones():
    """An item of far more parts than the others, which the merge joins, with one and more KV heads."""
    for hkv in (1, 2, 8):
        run([70, 30, 40, 300, 9000, 61, 0, 90], [3, 9, 1, 4, 5, 2, 8, 3], 4 * hkv, hkv)


def test_chains_of_many_tokens():
    """Without a mask a request may have any number of nodes: a prompt's."""
    run([77, 0], [700, 1100], 2, 1, "chain")


def test_requests_without_nodes_around_the_others():
    """More than 64 of them at a time, before, between and after those that have any."""
    rng = np.random.default_rng(3)
    nodes, prior = np.zeros(420, int), rng.integers(0, 50, size=420)
    for b, n, p in ((70, 3, 5000), (71, 9, 0), (200, 1, 16), (333, 40, 9000)):
        nodes[b], prior[b] = n, p
    run(prior.tolist(), nodes.tolist(), 4, 2)
    run(prior.tolist(), nodes.tolist(), 4, 2, "chain", lse=False)


def test_rows_before_the_first_request():
    """row_starts need not begin at 0; the rows before are left as they were."""
    s = Step([100, 2000, 3], [5, 70, 9], 8, 2, padding=7)
    s.call()
    s.check()
    want, want_lse = s.out[:84].clone(), s.lse[:84].clone()
    s.q, s.mask = s.q.roll(4, 0), s.mask.roll(4, 0)
    s.starts += 4
    s.out.fill_(5.0), s.lse.fill_(5.0)
    s.call()
    torch.cuda.synchronize()
    assert torch.equal(s.out[4:88].view(torch.int16), want.view(torch.int16)) and torch.equal(s.lse[4:88], want_lse)
    for t in (s.out, s.lse):
        assert (t[:4] == 5.0).all() and (t[88:] == 5.0).all()
    s.close()


class Coded:
    """Chains of `nodes` over a cache of coded pages."""

    def __init__(self, prior, nodes, hq, hkv, seed):
        rng = np.random.default_rng(seed)
        self.prior, self.nodes, self.hq, self.hkv = prior, nodes, hq, hkv
        B = len(prior)
        self.pages = -(-(prior + nodes) // 16)
        pool = int(self.pages.sum()) + 5
        perm, at = rng.permutation(pool), 0
        table = np.full((B, int(self.pages.max())), 2 ** 30)
        key, value = (np.full((pool, hkv), -1) for _ in "kv")
        for b, n in enumerate(self.pages):
            table[b, :n] = perm[at:at + n]
            at += n
            for g in range(hkv):
                key[table[b, :n], g], value[table[b, :n], g] = tree_codes.codes(b, g, int(n))
        caches = []
        for code, size in ((key, tree_codes.KEY), (value, tree_codes.VALUE)):
            x = torch.full((pool, hkv, 16, 128), float("nan"), dtype=torch.bfloat16, device="cuda")  # unused pages
            c = torch.from_numpy(code).cuda()
            used = torch.from_numpy(np.unique(table[table < 2 ** 30])).cuda()
            hot = (c[used][..., None] == torch.arange(128, device="cuda")).bfloat16() * size
            x[used] = hot[:, :, None, :].expand(-1, -1, 16, -1)
            caches.append(x)
        self.k, self.v = (torch.empty(pool * hkv * 2048, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        self.layout = libra.libra_kv_layout_create(self.k, self.v, pool, hkv)
        libra.libra_kv_pack_pages(self.layout, *caches, 0, pool)
        self.rows = B * nodes
        g = torch.Generator().manual_seed(seed)
        self.q = torch.randn((self.rows, hq, 128), generator=g).bfloat16().cuda()
        self.table = torch.from_numpy(table.astype(np.int32)).cuda()
        self.starts = torch.arange(B + 1, dtype=I32, device="cuda") * nodes
        self.dprior = torch.from_numpy(prior.astype(np.int32)).cuda()
        self.ws = torch.full((libra.libra_tree_attn_workspace_bytes(self.rows, B, hq, hkv),), 255, dtype=torch.uint8,
                             device="cuda")

    def call(self):
        out = torch.full_like(self.q, float("nan"))
        lse = torch.full(self.q.shape[:2], float("nan"), device="cuda")
        libra.libra_tree_attn(self.layout, self.q, self.dprior, self.starts, None, self.table, self.table.shape[1],
                              self.hq, SCALE, self.ws, out, lse)
        torch.cuda.synchronize()
        return out, lse

    def check(self, out, lse):
        out, lse, q, n, G = f64(out), f64(lse), f64(self.q), self.nodes, self.hq // self.hkv
        for b, prior in enumerate(self.prior):
            for g in range(self.hkv):
                r, h = slice(b * n, (b + 1) * n), slice(g * G, (g + 1) * G)
                key, value = tree_codes.codes(b, g, int(self.pages[b]))
                want, want_lse, score = tree_codes.attention(q[r, h], int(prior), key, value, SCALE)
                tol, lse_tol = tree_codes.tolerances(want, prior + n, score)
                assert (np.abs(out[r, h] - want) <= tol + 1e-30).all(), (b, g)
                assert (np.abs(lse[r, h] - want_lse) <= lse_tol).all(), (b, g)

    def close(self):
        libra.libra_kv_layout_destroy(self.layout)


@pytest.mark.parametrize("nodes", [1, 9, 50, 64, 65, 130])
def test_every_page_of_long_ranges(nodes):
    """Workgroups take several hundred steps, so several turns of staged page ids, in each form."""
    prior = np.random.default_rng(nodes).integers(1000, 30000 if nodes < 100 else 12000, size=48)
    s = Coded(prior, nodes, 8, 4, nodes)
    out, lse = s.call()
    s.check(out, lse)
    s.close()


@pytest.mark.parametrize("prior", [[131072], [126000, 3, 4000], [60000] * 5])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (16, 2), (28, 4)])
def test_every_page_of_few_long_contexts(prior, hq, hkv):
    """Items that many workgroups share, whose parts the merge joins."""
    s = Coded(np.array(prior), 5, hq, hkv, 3)
    out, lse = s.call()
    s.check(out, lse)
    s.close()


def test_a_captured_step_follows_its_lengths():
    """Pages, normalised keys, attention and accepted tokens of a step in one graph, replayed over steps of other
    lengths, masks and values, with eager work between: each replay gives the eager calls' bits."""
    rng = np.random.default_rng(11)
    B, hq, hkv, columns, most, rows = 6, 8, 2, 60, 4, 40
    pool = B * columns
    rot = libra.libra_rotary_create(base=1e6)
    wq, wk = (1 + 0.2 * torch.randn((2, 128), device="cuda")).bfloat16()
    zeros = lambda *n: torch.zeros(n, dtype=I32, device="cuda")

    class Side:
        def __init__(self):
            self.cache = Cache(pool, hkv)
            self.prior, self.new, self.held, self.table = zeros(B), zeros(B), zeros(B), zeros(B, columns)
            self.free, self.num_free = torch.arange(pool, dtype=I32, device="cuda"), zeros(1) + pool
            self.depths, self.slots, self.positions = zeros(rows), zeros(rows).long(), zeros(rows)
            self.starts, self.refused, self.mask = zeros(B + 1), zeros(B), zeros(rows, 1)
            self.accepted, self.counts = zeros(B, most), zeros(B)
            self.qkv = torch.zeros((rows, hq + 2 * hkv, 128), dtype=torch.bfloat16, device="cuda")
            self.q_out, self.out = (torch.zeros((rows, hq, 128), dtype=torch.bfloat16, device="cuda") for _ in "qo")
            self.lse = torch.zeros((rows, hq), device="cuda")
            self.ws = torch.zeros(libra.libra_tree_attn_workspace_bytes(rows, B, hq, hkv), dtype=torch.uint8,
                                  device="cuda")

        def step(self):
            q, k, v = self.qkv.split([hq, hkv, hkv], dim=1)
            libra.libra_kv_map(self.prior, self.new, self.held, self.table, columns, self.free, self.num_free,
                               self.depths, self.slots, self.positions, self.starts, self.held, self.num_free,
                               self.refused)
            libra.libra_kv_append_norm(self.cache.layout, rot, self.positions, self.slots, q, k, v, wq, wk, 1e-6,
                                       self.q_out)
            libra.libra_tree_attn(self.cache.layout, self.q_out, self.prior, self.starts, self.mask, self.table,
                                  columns, hq, SCALE, self.ws, self.out, self.lse)
            libra.libra_kv_accept(self.cache.layout, self.prior, self.accepted, self.counts, self.table, columns)

        def state(self):
            torch.cuda.synchronize()
            k, v = self.cache.logical()
            return [k.view(torch.int16), v.view(torch.int16), self.out.view(torch.int16), self.lse.view(I32),
                    self.q_out.view(torch.int16), self.slots, self.positions, self.starts, self.held, self.table,
                    self.num_free, self.refused]

    eager, replayed = Side(), Side()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.step()
    prior = np.zeros(B, int)
    for turn in range(8):
        new = rng.integers(1, 7, size=B) if turn else np.full(B, 6)
        if turn == 4:
            prior[2] = 0                                  # another request in its place
        seen = [tree_masks(rng, int(n), "tree") for n in new]
        bits, depths, accepted, counts = np.zeros((rows, 32), bool), np.zeros(rows), np.zeros((B, most)), np.zeros(B)
        at = np.concatenate([[0], np.cumsum(new)])
        for b in range(B):
            bits[at[b]:at[b + 1], :new[b]] = seen[b]
            depths[at[b]:at[b + 1]] = seen[b].sum(axis=1) - 1
            path = np.flatnonzero(seen[b][-1])[:most]
            accepted[b, :len(path)], counts[b] = path, len(path)
        words = np.packbits(bits, axis=1, bitorder="little").view(np.int32)
        values = torch.from_numpy(rng.standard_normal((rows, hq + 2 * hkv, 128))).bfloat16()
        for s in (eager, replayed):
            for t, a in ((s.prior, prior), (s.new, new), (s.mask, words), (s.depths, depths),
                         (s.accepted, accepted), (s.counts, counts)):
                t.copy_(torch.from_numpy(np.asarray(a)).to(I32))
            s.qkv.copy_(values)
        eager.step()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(eager.state(), replayed.state())), turn
        assert not eager.refused.any()
        live = f64(eager.lse)[:int(new.sum())]
        assert np.isfinite(live).all()
        prior = prior + counts.astype(int) + (150 if turn == 0 else 0)  # and some tokens of nothing
    libra.libra_rotary_destroy(rot)
    eager.cache.close()
    replayed.cache.close()
