"""libra_tree_attn on the GPU against the float64 oracle.

Tolerances.  A score adds 128 bf16 products in float32: off by e = 140 2^-24 of scale * sum |q k|; a
probability by 2 e of itself, by the exp2's 2^-22, and by 2^-8 once it is rounded to bf16; the output by
that much of A = sum p |v|, by as much again for the sums over keys ((n / 32 + 60) 2^-24), and by its own
rounding, 2^-8.  The log-sum-exp: e, the sums, and float32's last bits."""
import numpy as np
import pytest
import torch

from oracle import drafts as ref
from paper_2606_03077_amd import libra

from test_gpu_kv_append import Cache

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))
I32 = torch.int32


def f64(t):
    return t.double().cpu().numpy()


def tree_masks(rng, n, kind):
    if kind == "chain":
        return np.tril(np.ones((n, n), bool))
    if kind == "any":                                  # bits that form no tree, some rows without any
        m = rng.random((n, n)) < 0.4
        m[rng.random(n) < 0.3] = False
        return m
    if kind == "none":
        return np.zeros((n, n), bool)
    m = np.zeros((n, n), bool)
    for i in range(n):
        p = int(rng.integers(-1, i)) if i else -1
        if p >= 0:
            m[i] = m[p]
        m[i, i] = True
    return m


class Step:
    """A call's arrays.  Everything that no row may see holds `junk`, and unused table entries too."""

    def __init__(self, prior, nodes, hq, hkv, kind="tree", seed=1, padding=3, scale_q=1.0, junk=float("nan"),
                 words=None):
        rng = np.random.default_rng(seed)
        self.prior, self.nodes, self.hq, self.hkv, self.kind = list(prior), list(nodes), hq, hkv, kind
        pages = [-(-(p + n) // 16) for p, n in zip(prior, nodes)]
        pool = sum(pages) + 3
        self.cache = Cache(pool, hkv, seed)
        perm, at = rng.permutation(pool), 0
        self.columns = max(pages + [1]) + 1
        table = np.full((len(prior), self.columns), 2 ** 30)
        kept = np.zeros(pool * 16, bool)
        for b, n in enumerate(pages):
            table[b, :n] = perm[at:at + n]
            at += n
            t = np.arange(prior[b] + nodes[b])
            kept[table[b, t // 16] * 16 + t % 16] = True
        k, v = self.cache.initial()
        gone = torch.from_numpy(~kept).cuda()
        k[gone] = junk
        v[gone] = junk
        self.set(k, v)
        rows = sum(nodes) + padding
        g = torch.Generator().manual_seed(seed)
        self.q = (torch.randn((rows, hq, 128), generator=g) * scale_q).bfloat16().cuda()
        self.seen = [tree_masks(rng, n, kind) for n in nodes]
        self.words = words or max(1, -(-max(nodes + [1]) // 32))
        bits = rng.random((rows, 32 * self.words)) < 0.5    # beyond a request's nodes: anything
        starts = np.concatenate([[0], np.cumsum(nodes)]).astype(int)
        for b, n in enumerate(nodes):
            m = min(n, 32 * self.words)
            bits[starts[b]:starts[b + 1], :m] = self.seen[b][:, :m]
            self.seen[b][:, m:] = False
        if kind == "chain":
            self.mask = None
        else:
            self.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
        self.table = torch.from_numpy(table.astype(np.int32)).cuda()
        self.host_table, self.start = table, starts
        self.dprior = torch.tensor(self.prior, dtype=I32, device="cuda")
        self.starts = torch.tensor(starts, dtype=I32, device="cuda")
        self.out = torch.full((rows, hq, 128), 5.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((rows, hq), 5.0, device="cuda")
        n = libra.libra_tree_attn_workspace_bytes(rows, len(prior), hq, hkv)
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def set(self, k, v):
        """The cache's logical content, [slots, hkv, 128]."""
        self.k, self.v = k, v
        page = lambda t: t.reshape(-1, 16, self.hkv, 128).transpose(1, 2).contiguous()
        libra.libra_kv_pack_pages(self.cache.layout, page(k), page(v), 0, self.cache.pages)

    def tokens(self, b):
        t = np.arange(self.prior[b] + self.nodes[b])
        at = torch.from_numpy(self.host_table[b, t // 16] * 16 + t % 16).cuda()
        return f64(self.k[at]), f64(self.v[at])

    def call(self, lse=True, stream=None):
        libra.libra_tree_attn(self.cache.layout, self.q, self.dprior, self.starts, self.mask, self.table,
                              self.columns, self.hq, SCALE, self.ws, self.out, self.lse if lse else None,
                              stream=stream)

    def check(self, lse=True, skip=None):
        """skip: a row that is not looked at."""
        torch.cuda.synchronize()
        out, got_lse, q = f64(self.out), f64(self.lse), f64(self.q)
        for b, n in enumerate(self.nodes):
            r = slice(self.start[b], self.start[b] + n)
            k, v = self.tokens(b)
            want, want_lse, size, score = ref.tree_attention(q[r], k, v, self.prior[b], self.seen[b], SCALE)
            if skip is not None and r.start <= skip < r.stop:
                i = skip - r.start
                want[i], want_lse[i], size[i], score[i] = out[skip], got_lse[skip], 0, 0
            e = 140 * 2.0 ** -24 * score
            sums = (len(k) / 32 + 60) * 2.0 ** -24
            tol = (2.0 ** -8 + 2 * e + sums + 2.0 ** -20)[..., None] * size + 1.01 * 2.0 ** -8 * np.abs(want)
            with np.errstate(invalid="ignore"):
                finite = np.isfinite(want)
                same = (out[r] == want) | (np.isnan(out[r]) & np.isnan(want))
                bad = np.where(finite, ~(np.abs(out[r] - want) <= tol + 1e-30), ~same)
                assert not bad.any(), (b, np.argwhere(bad)[:5], out[r][bad][:5], want[bad][:5])
                if lse:
                    tol = e + sums + 2.0 ** -21 * (1 + np.abs(want_lse))
                    bad = ~((np.abs(got_lse[r] - want_lse) <= tol) | (got_lse[r] == want_lse)
                            | (np.isnan(got_lse[r]) & np.isnan(want_lse)))
                    assert not bad.any(), (b, got_lse[r][bad][:5], want_lse[bad][:5])
        end = self.start[-1]
        assert (self.out[end:] == 5.0).all() and (self.lse[end:] == 5.0).all()
        if not lse:
            assert (self.lse == 5.0).all()

    def close(self):
        self.cache.close()


def run(*args, lse=True, **kw):
    s = Step(*args, **kw)
    s.call(lse)
    s.check(lse)
    s.close()


@pytest.mark.parametrize("kind", ["tree", "chain", "any", "none"])
@pytest.mark.parametrize("prior,nodes", [
    ([0], [1]), ([1], [1]), ([0], [5]), ([15], [1]), ([16], [2]), ([31], [2]), ([32], [33]), ([1000], [7]),
    ([500, 3, 0, 77], [4, 1, 9, 16]), ([64, 64], [32, 32]), ([5, 900, 0, 40], [0, 3, 0, 2])])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 4), (16, 1)])
def test_small_trees(kind, prior, nodes, hq, hkv):
    run(prior, nodes, hq, hkv, kind)


@pytest.mark.parametrize("kind", ["tree", "any", "chain"])
@pytest.mark.parametrize("nodes,hq,hkv", [(64, 4, 1), (130, 2, 1), (200, 7, 1), (256, 3, 1), (100, 28, 4)])
def test_wide_trees(kind, nodes, hq, hkv):
    """Several tiles of every form, masks of up to eight words."""
    run([100, 33], [nodes, max(1, nodes - 3)], hq, hkv, kind)


@pytest.mark.parametrize("prior", [2000, 6001, 20000])
@pytest.mark.parametrize("nodes,hq,hkv", [(3, 4, 2), (9, 7, 1), (1, 8, 8)])
def test_long_contexts_are_split(prior, nodes, hq, hkv):
    run([prior, 40], [nodes, nodes], hq, hkv)


@pytest.mark.parametrize("form", [1, 2, 4, 8])  # 32, 64, 128, 256 rows
def test_one_long_among_many(form):
    """Each form of the kernel; workgroups that end one request's item and begin the next's."""
    rng = np.random.default_rng(form)
    nodes = [8 * form] * 20
    nodes[3] = 1
    run(rng.integers(0, 300, size=19).tolist() + [4000], nodes, 8, 2)


def test_many_requests():
    rng = np.random.default_rng(5)
    run(rng.integers(0, 40, size=700).tolist(), rng.integers(0, 4, size=700).tolist(), 2, 1)


def test_uneven_trees():
    """A request with far more rows than the average that chose the form."""
    run([50] * 12 + [900], [1] * 12 + [120], 4, 1)


def test_mask_words_beyond_and_below_the_nodes():
    run([20, 40], [6, 40], 4, 2, words=8)
    run([20, 40], [6, 40], 4, 2, kind="any", words=1)   # nodes past the words are seen by none


def test_without_lse():
    run([100, 2000], [5, 6], 8, 2, lse=False)


def test_no_nodes_at_all():
    s = Step([10, 20], [0, 0], 4, 2)
    s.call()
    s.check()
    s.close()


@pytest.mark.parametrize("scale_q", [0.01, 30.0])
def test_score_ranges(scale_q):
    run([700, 50], [9, 20], 8, 2, scale_q=scale_q)


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -3e38])
def test_unseen_nodes_may_hold_anything(junk):
    """Nodes that most rows do not see have keys and values that are not finite: a row that does not
    see one is as without it, a row that sees an infinite value has it."""
    for kind in ("tree", "any"):
        s = Step([40, 70, 0], [12, 40, 33], 8, 2, kind, junk=junk)
        k, v = s.k.clone(), s.v.clone()
        for b, node in ((0, 3), (1, 20), (1, 39), (2, 1)):
            t = s.prior[b] + node
            at = int(s.host_table[b, t // 16]) * 16 + t % 16
            v[at, :, ::2] = junk
            s.seen[b][:, node] &= np.arange(s.nodes[b]) == node  # its own row only
        starts = s.start
        bits = np.zeros((s.q.shape[0], 32 * s.words), bool)
        for b, n in enumerate(s.nodes):
            bits[starts[b]:starts[b + 1], :n] = s.seen[b]
        s.mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
        s.set(k, v)
        s.call()
        s.check()
        # Keys too.  Rows that do not see one are within the same tolerances, but not the same bits as
        # before: a wave's 32 rows move their maxima together, and a NaN score moves them, which changes
        # what the probabilities are rounded at (a power of two times the moved maximum's fraction).
        t = s.prior[1] + 20
        k[int(s.host_table[1, t // 16]) * 16 + t % 16] = junk
        s.set(k, v)
        s.call()
        s.check(skip=starts[1] + 20)
        s.close()


def test_nan_and_infinite_context():
    s = Step([400, 40], [4, 4], 4, 2)
    k, v = s.k.clone(), s.v.clone()
    at = int(s.host_table[0, 5]) * 16 + 3
    v[at, 0, 7], v[at, 1, 9] = float("inf"), float("nan")
    s.set(k, v)
    s.call()
    torch.cuda.synchronize()
    out = s.out.view(-1, 2, 2, 128)
    assert (out[:4, 0, :, 7] == float("inf")).all() and out[:4, 1, :, 9].isnan().all()
    assert out[:4, 0, :, :7].isfinite().all() and out[4:8].isfinite().all()
    s.close()


def test_table_ids_outside_the_cache_and_short_tables():
    """What a refused request leaves behind: no fault, and the other requests' rows are right."""
    s = Step([100, 200, 50], [3, 3, 3], 4, 2, padding=0)
    good = s.table.clone()
    s.call()
    torch.cuda.synchronize()
    want = s.out.clone()
    s.table[1] = torch.tensor([-1, 2 ** 30, 2 ** 31 - 1, -2 ** 31] * 9, dtype=I32)[:s.columns]
    s.call()
    torch.cuda.synchronize()
    keep = [0, 1, 2, 6, 7, 8]
    assert torch.equal(s.out[keep].view(torch.int16), want[keep].view(torch.int16))
    s.table.copy_(good)
    s.dprior[1] = 2 ** 31 - 1                            # tokens past the table are not seen
    s.call()
    torch.cuda.synchronize()
    s.dprior[1] = -7
    s.call()
    torch.cuda.synchronize()
    s.dprior[1] = 200
    s.starts[3] = 10 ** 6                               # rows past the end are not there
    s.call()
    s.check()
    s.close()


def test_replays_follow_lengths_masks_and_tables():
    """One captured call serves other lengths in the same memory, with eager work between, and shares its
    workspace with another graph."""
    a = Step([3000, 10, 500], [4, 7, 5], 8, 2, seed=3)
    b = Step([20, 2500, 1], [6, 2, 8], 8, 2, seed=4)
    assert a.ws.numel() == b.ws.numel()
    b.ws = a.ws
    graphs = []
    for s in (a, b):
        s.call()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.call()
        graphs.append(g)
    for turn in range(3):
        for s, g in zip((a, b), graphs):
            s.out.fill_(5.0)
            s.lse.fill_(5.0)
            g.replay()
            s.check()
            first = s.out.clone()
            s.call()                                     # equal calls, equal bits
            torch.cuda.synchronize()
            assert torch.equal(first.view(torch.int16), s.out.view(torch.int16))
        # Shorter contexts in the first graph's memory.
        a.prior = [max(0, p - 100 * (turn + 1)) for p in a.prior]
        k, v = a.k.clone(), a.v.clone()
        a.dprior.copy_(torch.tensor(a.prior, dtype=I32))
        a.set(k, v)
    a.close()
    b.close()


def test_on_another_stream():
    s = Step([100, 900], [5, 6], 8, 2)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    s.call(stream=stream)
    stream.synchronize()
    s.check()
    s.close()


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    steps = [Step([3000, 70, 900], [9, 3, 30], 8, 2, seed=1), Step([500] * 20, [40] * 20, 8, 2, "any", seed=2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, s in zip(steps, streams):
            t.call(stream=s)
    for t in steps:
        t.check()


def test_one_node_is_a_decode_step():
    """Single tokens give what libra_decode_attn gives over the same cache, to both sides' rounding."""
    prior = [700, 16, 3001, 0]
    s = Step(prior, [1] * 4, 8, 2, kind="chain", padding=0)
    s.call()
    plan = libra.libra_splitkv_plan(libra.LIBRA_MODE_DECODE, 4, 8, 2, [p + 1 for p in prior], None)
    out, lse = torch.zeros_like(s.out), torch.zeros_like(s.lse)
    libra.libra_decode_attn(s.cache.layout, plan, s.q, s.table, s.columns, 4, 8, SCALE,
                            libra.alloc_workspace(plan), out, lse)
    s.check()
    libra.libra_plan_destroy(plan)
    # Each within 2^-8 of sum p |v| (about 0.8 for N(0, 1) values) and of itself from the exact one.
    assert (out.float() - s.out.float()).abs().max() <= 4 * 2.0 ** -8 * max(1.0, float(out.abs().max()))
    assert (lse - s.lse).abs().max() <= 1e-4
    s.close()


def test_a_drafted_step():
    """The operators as a step uses them: pages, normalised keys, attention, accepted tokens, pages back."""
    rng = np.random.default_rng(7)
    B, hq, hkv, columns = 5, 8, 2, 20
    pool = B * columns
    cache = Cache(pool, hkv)
    rot = libra.libra_rotary_create(base=1e6)
    dev = lambda a, dtype=I32: torch.as_tensor(np.asarray(a), dtype=dtype).cuda()
    zeros = lambda *n: torch.zeros(n, dtype=I32, device="cuda")
    prior, new = rng.integers(20, 200, size=B), rng.integers(1, 9, size=B)
    held, table, free, num_free = zeros(B), zeros(B, columns), dev(rng.permutation(pool)), dev([pool])
    starts, refused = zeros(B + 1), zeros(B)
    wq, wk = (1 + 0.2 * torch.randn((2, 128), device="cuda")).bfloat16()

    def step(prior, new, depths):
        """Maps and appends `new` tokens behind `prior`; the turned queries, keys, values and their slots."""
        rows = int(new.sum()) + 2
        slots, positions = torch.zeros(rows, dtype=torch.int64, device="cuda"), zeros(rows)
        libra.libra_kv_map(dev(prior), dev(new), held, table, columns, free, num_free, depths, slots,
                           positions, starts, held, num_free, refused)
        qkv = torch.randn((rows, hq + 2 * hkv, 128), device="cuda").bfloat16()
        q, k, v = qkv.split([hq, hkv, hkv], dim=1)
        q_out, k_out = torch.zeros_like(q).contiguous(), torch.zeros_like(k).contiguous()
        libra.libra_kv_append_norm(cache.layout, rot, positions, slots, q, k, v, wq, wk, 1e-6, q_out)
        libra.libra_qk_norm_rotary(rot, k, None, wk, None, 1e-6, positions, k_out, None)
        assert not refused.any()
        return q_out, k_out, v, slots

    _, k0, v0, _ = step(np.zeros(B, int), prior, None)
    at = np.concatenate([[0], np.cumsum(prior)])
    context = [(k0[at[b]:at[b + 1]], v0[at[b]:at[b + 1]]) for b in range(B)]
    seen = [tree_masks(rng, int(n), "tree") for n in new]
    rows = int(new.sum()) + 2
    bits = np.zeros((rows, 32), bool)
    depths = np.zeros(rows, int)
    at = np.concatenate([[0], np.cumsum(new)])
    for b in range(B):
        bits[at[b]:at[b + 1], :new[b]] = seen[b]
        depths[at[b]:at[b + 1]] = seen[b].sum(axis=1) - 1
    q, k, v, slots = step(prior, new, dev(depths))
    mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
    ws = torch.zeros(libra.libra_tree_attn_workspace_bytes(rows, B, hq, hkv), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((rows, hq), device="cuda")
    libra.libra_tree_attn(cache.layout, q, dev(prior), starts, mask, table, columns, hq, SCALE, ws, out, lse)
    paths = [np.flatnonzero(seen[b][-1]) for b in range(B)]    # the last node's ancestors and itself
    accepted = np.zeros((B, 8), int)
    for b, p in enumerate(paths):
        accepted[b, :len(p)] = p
    counts = np.array([len(p) for p in paths])
    libra.libra_kv_accept(cache.layout, dev(prior), dev(accepted), dev(counts), table, columns)
    torch.cuda.synchronize()
    logical = cache.logical()
    for b in range(B):
        r = slice(at[b], at[b + 1])
        ks, vs = (torch.cat([context[b][i], (k, v)[i][r]]) for i in (0, 1))
        want, want_lse, size, score = ref.tree_attention(f64(q[r]), f64(ks), f64(vs), int(prior[b]), seen[b], SCALE)
        e = 140 * 2.0 ** -24 * score
        tol = (2.0 ** -8 + 2 * e + 2.0 ** -16)[..., None] * size + 1.01 * 2.0 ** -8 * np.abs(want)
        assert (np.abs(f64(out[r]) - want) <= tol).all()
        assert (np.abs(f64(lse[r]) - want_lse) <= e + 2.0 ** -16 * (1 + np.abs(want_lse))).all()
        n = int(prior[b]) + len(paths[b])
        t = torch.arange(n, device="cuda")
        slot = table[b, t // 16].long() * 16 + t % 16
        for got, full in zip(logical, (ks, vs)):
            keep = torch.cat([full[:int(prior[b])], full[int(prior[b]) + torch.from_numpy(paths[b]).cuda()]])
            assert torch.equal(got[slot], keep)
    step(prior + counts, np.zeros(B, int), None)
    torch.cuda.synchronize()
    assert held.tolist() == [-(-int(n) // 16) for n in prior + counts]
    assert int(held.sum()) + int(num_free) == pool
    libra.libra_rotary_destroy(rot)
    cache.close()


@pytest.mark.parametrize("nodes", [1, 6, 20, 50])
def test_large_batches_against_append_attention(nodes):
    """Chains over so many tokens that a workgroup's range goes on for several turns of page ids, in every
    form, against libra_append_attn (which writes the tokens that are there): both within 2^-8 of sum p |v|
    (at most the largest |v|) and of themselves, twice."""
    rng = np.random.default_rng(nodes)
    B, hq, hkv = 70, 8, 4
    lens = rng.integers(1000, 30000, size=B)
    pages = -(-lens // 16)
    pool = int(pages.sum())
    g = torch.Generator(device="cuda").manual_seed(nodes)
    k, v = (torch.randn((pool * hkv * 2048,), device="cuda", generator=g, dtype=torch.bfloat16) for _ in "kv")
    layout = libra.libra_kv_layout_create(k, v, pool, hkv)
    perm, at = rng.permutation(pool), 0
    table = np.zeros((B, int(pages.max())), np.int32)
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    starts = torch.arange(B + 1, dtype=I32, device="cuda") * nodes
    rows = B * nodes
    q = torch.randn((rows, hq, 128), device="cuda", generator=g).bfloat16()
    bt = torch.from_numpy(table).cuda()
    ws = torch.empty(libra.libra_tree_attn_workspace_bytes(rows, B, hq, hkv), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((rows, hq), device="cuda")
    prior = torch.tensor((lens - nodes).tolist(), dtype=I32, device="cuda")
    libra.libra_tree_attn(layout, q, prior, starts, None, bt, table.shape[1], hq, SCALE, ws, out, lse)
    # The new tokens as they are, gathered.
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=I32, device="cuda")
    ks, vs = (torch.empty((int(lens.sum()), hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    libra.libra_kv_gather(layout, bt, table.shape[1], cu, B, table.shape[1], ks, vs)
    new = torch.cat([torch.arange(int(e) - nodes, int(e)) for e in np.cumsum(lens)]).cuda()
    plan = libra.libra_splitkv_plan(libra.LIBRA_MODE_APPEND, B, hq, hkv, lens.tolist(), [nodes] * B)
    want, want_lse = torch.empty_like(q), torch.empty_like(lse)
    libra.libra_append_attn(layout, plan, q, ks[new].contiguous(), vs[new].contiguous(), bt, table.shape[1], B, hq,
                            SCALE, libra.alloc_workspace(plan), want, want_lse)
    torch.cuda.synchronize()
    libra.libra_plan_destroy(plan)
    tol = 2 * 2.0 ** -8 * (1 + want.float().abs())  # sum p |v| over a thousand keys or more is about 0.8
    assert ((out.float() - want.float()).abs() <= tol).all()
    assert ((lse - want_lse).abs() <= 1e-3).all()
    again = torch.empty_like(out)
    libra.libra_tree_attn(layout, q, prior, starts, None, bt, table.shape[1], hq, SCALE, ws, again, None)
    torch.cuda.synchronize()
    libra.libra_kv_layout_destroy(layout)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))
