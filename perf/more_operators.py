"""Performance cases of a drafted step over the paged cache: block tables and slots built from
request lengths on the GPU, norms of queries and keys with their rotary positions (on the way
into the cache, and with gradients), attention of a tree of drafted tokens, and the move of the
accepted tokens into place.

Each case is a dict of plain values.  ``prepare`` makes what a program holds before the call,
``run`` makes one pass, ``exact`` gives the same outputs in float64.  With ``own`` false ``run``
computes the operators from elementary torch operations; with ``own`` true it calls the library.

Tables ("map"): request b holds ``held`` pages of its row of the block table and wants
ceil((prior + new) / 16).  Surplus pages go back on top of the stack of free pages (requests, then
pages, in ascending order), then missing ones are taken from its top; a request whose pages, with
those of all before it, exceed the stack is refused and keeps what it has.  New row r of request b
is token prior + i: its slot is page * 16 + token % 16, its position prior + depth (or + i).

Norm ("append", "train"): n = x / sqrt(mean(x^2) + eps) over a head's channels, u = w n, y = u
turned by the row's position: pairs j of the first R channels by position * theta_j, theta_j =
base^(-2 j / R); channels (j, j + R / 2) in the half layout, (2 j, 2 j + 1) in the interleaved one.

Trees ("tree"): node i of request b attends its ``prior`` cached tokens and those nodes of the
request (cached behind them) whose bits are set in its mask, itself and its ancestors; without a
mask, every earlier node and itself.

Accepted tokens ("accept"): node ``accepted[b][i]``'s K and V move to token prior + i.

Cache tiles (page, KV head) hold 16 slots x 128 channels; K as [16 channel blocks][16 slots][8],
V as [slot / 4 % 2][128 channels][slot / 8][slot % 4].

Lengths, trees and positions come from the case alone (``shape`` seeds them), values and page
placement from the seed.  Values are N(0, 1) in the tensors' type, norm weights 1 + 0.2 N(0, 1).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
DIM = 128
SCALE = float(np.float32(1.0 / math.sqrt(DIM)))
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# --- the cases -------------------------------------------------------------------------

def _lens(batch, lens, mid, lo, hi):
    return {"batch": batch, "lens": lens, "mid": mid, "lo": lo, "hi": hi}


def listed():
    return [
        # The pages and slots of a decode step of 64 requests: latency.
        {"name": "map_step", "op": "map", **_lens(64, "lognormal", 2048, 64, 32768), "new_lo": 1,
         "new_hi": 1, "depths": False, "ended": 0, "short": False, "padding": 0, "shape": 26062},
        # The drafted trees of 256 requests, of which some have ended and give their pages back;
        # the rows are padded to a captured graph's size.
        {"name": "map_trees", "op": "map", **_lens(256, "lognormal", 4096, 256, 32768),
         "new_lo": 1, "new_hi": 64, "depths": True, "ended": 9, "short": False, "padding": 301,
         "shape": 26063},
        # Keys, values and queries of a decode step, 16 requests of the 40/8-head shape: latency.
        {"name": "append_step", "op": "append", "hq": 40, "hkv": 8, "rows": 16, "run": 1,
         "padding": 0, "rdim": 128, "layout": "half", "base": 1000000.0, "shape": 11},
        # Of 32 ragged prompts and tool outputs, padded.
        {"name": "append_chunks", "op": "append", "hq": 40, "hkv": 8, "rows": 16381, "run": 512,
         "padding": 77, "rdim": 128, "layout": "half", "base": 1000000.0, "shape": 12},
        # A training pass over short responses, float32, interleaved pairs in half of each head.
        {"name": "train_fp32", "op": "train", "hq": 28, "hkv": 4, "dim": 128, "rows": 2003,
         "type": "fp32", "rdim": 64, "layout": "interleaved", "base": 10000.0, "shape": 13},
        # A training pass over a micro-batch of long responses.
        {"name": "train_bf16", "op": "train", "hq": 40, "hkv": 8, "dim": 128, "rows": 16381,
         "type": "bf16", "rdim": 128, "layout": "half", "base": 1000000.0, "shape": 14},
        # A small model's drafts for a few short requests.
        {"name": "tree_small", "op": "tree", "hq": 8, "hkv": 2, **_lens(8, "uniform", 0, 16, 512),
         "nodes_lo": 7, "nodes_hi": 7, "mask": True, "padding": 0, "shape": 26061},
        # An ordinary step of a 7B-class model: 64 requests, small trees of uneven size.
        {"name": "tree_7b", "op": "tree", "hq": 28, "hkv": 4,
         **_lens(64, "lognormal", 2048, 64, 32768), "nodes_lo": 5, "nodes_hi": 16, "mask": True,
         "padding": 33, "shape": 26062},
        # Wide trees, where the products weigh as much as the reads.
        {"name": "tree_wide", "op": "tree", "hq": 32, "hkv": 8,
         **_lens(32, "lognormal", 4096, 256, 32768), "nodes_lo": 64, "nodes_hi": 64, "mask": True,
         "padding": 0, "shape": 26064},
        # The straggler bucket: four long requests with chains of four drafted tokens.
        {"name": "tree_straggler", "op": "tree", "hq": 64, "hkv": 8,
         **_lens(4, "uniform", 0, 98304, 131072), "nodes_lo": 4, "nodes_hi": 4, "mask": False,
         "padding": 0, "shape": 4},
        # The accepted tokens of a few requests: latency.
        {"name": "accept_small", "op": "accept", "hkv": 4,
         **_lens(16, "lognormal", 2048, 64, 8192), "most": 4, "nodes": 16, "shape": 21},
        # Of a full batch, paths of up to 16 tokens.
        {"name": "accept_large", "op": "accept", "hkv": 8,
         **_lens(256, "lognormal", 1024, 64, 4096), "most": 16, "nodes": 64, "shape": 22},
    ]


HEADS = [(8, 2), (28, 4), (32, 8), (64, 8), (40, 8), (14, 2), (20, 4), (8, 1), (16, 4), (16, 1),
         (12, 4), (8, 8)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges: any operator, sizes spread over their logarithm."""
    op = rng.choice(["map", "append", "train", "tree", "tree", "accept"])
    shape = rng.randrange(1 << 30)
    hq, hkv = rng.choice(HEADS)
    if op == "map":
        hi, new = _log(rng, 64, 32768), _log(rng, 1, 512)
        batch = min(_log(rng, 1, 512), max(1, 2 * 16384 // new))
        return {"op": op, **_lens(batch, "lognormal", max(1, hi // 8), 0, hi),
                "new_lo": rng.choice([0, 1]), "new_hi": new, "depths": rng.random() < 0.5,
                "ended": rng.choice([0, batch // 8, batch // 2]), "short": rng.random() < 0.25,
                "padding": rng.choice([1, 2, 99]), "shape": shape}
    rope = {"rdim": rng.choice([128, 128, 64, 32, 96, 20]),
            "layout": rng.choice(["half", "interleaved"]), "base": rng.choice([1e4, 5e5, 1e6])}
    if op == "append":
        return {"op": op, "hq": rng.choice([hq, hq, hq, 0]), "hkv": hkv,
                "rows": min(_log(rng, 1, 16381), 786000 // (hq + hkv)),
                "run": rng.choice([1, 7, 33, 512]), "padding": rng.choice([0, 0, 1, 77]), **rope,
                "shape": shape}
    if op == "train":
        dim = rng.choice([128, 128, 128, 64, 256, 80])
        rope["rdim"] = min(rope["rdim"], dim - dim % 32)
        kind = rng.choice(list(TYPES))
        most = 50000000 if kind == "fp32" else 100000000
        return {"op": op, "hq": hq, "hkv": rng.choice([hkv, hkv, hkv, 0]), "dim": dim,
                "rows": min(_log(rng, 1, 16381), most // (dim * (hq + hkv))), "type": kind, **rope,
                "shape": shape}
    if op == "tree":
        hi, nodes = _log(rng, 64, 131072), _log(rng, 1, 128)
        batch = _log(rng, 1, 256)
        batch = min(batch, max(1, int(2e9 / (512 * hkv * hi))),
                    max(1, int(1e11 / (512 * hq * nodes * hi))))
        return {"op": op, "hq": hq, "hkv": hkv, **_lens(batch, "lognormal", max(1, hi // 4), 1, hi),
                "nodes_lo": rng.choice([1, max(1, nodes // 2), nodes]), "nodes_hi": nodes,
                "mask": rng.random() < 0.75, "padding": rng.choice([0, 0, 5]), "shape": shape}
    hi, most = _log(rng, 64, 4096), _log(rng, 1, 16)
    return {"op": op, "hkv": hkv, **_lens(_log(rng, 1, 256), "lognormal", hi // 4, 0, hi),
            "most": most, "nodes": min(256, 2 * most + _log(rng, 1, 128)), "shape": shape}


# --- sizes -----------------------------------------------------------------------------

def _prior(case, rng):
    B, lo, hi = case["batch"], case["lo"], case["hi"]
    if case["lens"] == "uniform":
        return rng.integers(lo, hi, size=B, endpoint=True).astype(np.int64)
    z = rng.standard_normal(B)
    return np.clip(np.rint(np.exp(math.log(case["mid"]) + z)), lo, hi).astype(np.int64)


def _pages(tokens):
    return (tokens + PAGE - 1) // PAGE


def _map_sizes(case):
    """(prior, new, held, depths): requests that ended want nothing and hold what they had."""
    rng = np.random.default_rng(case["shape"])
    prior = _prior(case, rng)
    new = rng.integers(case["new_lo"], case["new_hi"], size=case["batch"], endpoint=True)
    held = _pages(prior)
    # Pages that rejected tokens left behind: one too many here and there.
    held = held + (rng.random(case["batch"]) < 0.1)
    gone = rng.permutation(case["batch"])[:case["ended"]]
    prior[gone], new[gone] = 0, 0
    rows = int(new.sum()) + case["padding"]
    return prior, new.astype(np.int64), held, rng.integers(0, 8, size=rows)


def _tree_sizes(case):
    """(prior, nodes, parents of each request's nodes)."""
    rng = np.random.default_rng(case["shape"])
    prior = _prior(case, rng)
    nodes = rng.integers(case["nodes_lo"], case["nodes_hi"], size=case["batch"], endpoint=True)
    parents = [[int(rng.integers(-1, i)) if i else -1 for i in range(int(n))] for n in nodes]
    return prior, nodes.astype(np.int64), parents


def _seen(case, parents):
    """[n, n] truth values: node i attends node j."""
    n = len(parents)
    if not case["mask"]:
        return np.tril(np.ones((n, n), bool))
    seen = np.zeros((n, n), bool)
    for i, p in enumerate(parents):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def _accept_sizes(case):
    """(prior, counts, accepted [batch, most]): a breadth-first tree's accepted path, whose nodes
    lie behind the tokens that the path will take, or already in their place."""
    rng = np.random.default_rng(case["shape"])
    prior = _prior(case, rng)
    most = case["most"]
    counts = rng.integers(1, most, size=case["batch"], endpoint=True)
    accepted = np.zeros((case["batch"], most), np.int64)
    for b in range(case["batch"]):
        path = np.sort(rng.permutation(np.arange(most, case["nodes"]))[:most])
        stay = int(rng.integers(0, 2))
        accepted[b, :len(path)] = path
        accepted[b, :stay] = np.arange(stay)
    return prior, counts.astype(np.int64), accepted


def _append_rows(case):
    """Slots (-1: padding) before pages are placed, and positions: runs of consecutive tokens."""
    rng = np.random.default_rng(case["shape"])
    token, position, at = [], [], 0
    while len(token) < case["rows"]:
        n = min(int(rng.integers(1, case["run"], endpoint=True)), case["rows"] - len(token))
        first, p = int(rng.integers(PAGE)), int(rng.integers(0, 20000))
        token += range(at * PAGE + first, at * PAGE + first + n)
        position += range(p, p + n)
        at += (first + n + PAGE - 1) // PAGE
    return np.asarray(token, np.int64), np.asarray(position, np.int64), at


def work(case):
    op = case["op"]
    if op == "map":
        prior, new, held, depths = _map_sizes(case)
        rows, B = len(depths), case["batch"]
        want = _pages(prior + new)
        moved = int(np.abs(want - held).sum())
        b = 4 * B * 3 + 4 * (B + 2 * B + 1) + 8 * moved + 12 * rows
        b += 4 * rows if case["depths"] else 0
        return {"bytes": float(b), "flops": 0.0}
    if op == "append":
        rows, hq, hkv = case["rows"], case["hq"], case["hkv"]
        n = rows * (hq + hkv)
        return {"bytes": float(2 * 256 * (n + rows * hkv) + 12 * rows),
                "flops": float(n * (4 * DIM + 3 * case["rdim"]))}
    if op == "train":
        n = case["rows"] * (case["hq"] + case["hkv"])
        size = torch.empty(0, dtype=TYPES[case["type"]]).element_size()
        return {"bytes": float(5 * n * case["dim"] * size + 4 * case["rows"]),
                "flops": float(n * (14 * case["dim"] + 6 * case["rdim"]))}
    if op == "accept":
        prior, counts, accepted = _accept_sizes(case)
        at = np.arange(case["most"])[None]
        moved = int(((accepted != at) & (at < counts[:, None])).sum())
        return {"bytes": float(moved * 2 * 512 * case["hkv"]), "flops": 0.0}
    prior, nodes, parents = _tree_sizes(case)
    hq, hkv, rows = case["hq"], case["hkv"], int(nodes.sum())
    seen = sum(int(_seen(case, p).sum()) for p in parents) + int((prior * nodes).sum())
    b = int((prior + nodes).sum()) * 512 * hkv + rows * hq * (256 + 256 + 4)
    b += 4 * int(_pages(prior + nodes).sum())
    b += rows * 4 * ((int(nodes.max()) + 31) // 32) if case["mask"] else 0
    return {"bytes": float(b), "flops": 4.0 * DIM * hq * seen}


# --- inputs ----------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, shape, dtype=torch.bfloat16):
    return torch.randn(shape, dtype=dtype, device="cuda", generator=gen)


def _weight(gen, dim, dtype):
    return (1.0 + 0.2 * _normal(gen, (dim,), torch.float32)).to(dtype)


def _placement(pages, seed):
    """Physical pages of each sequence: (pool size, block table [B, columns], int32)."""
    need = int(pages.sum())
    pool = need + max(1, need // 100)
    perm = np.random.default_rng(int(seed)).permutation(pool).astype(np.int32)
    table = np.full((len(pages), max(1, int(pages.max()))), perm[need], np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += int(n)
    return pool, table


def _free_stack(case, seed):
    """(block table, free pages [pool], their number) before a call of "map"."""
    prior, new, held, depths = _map_sizes(case)
    want = _pages(prior + new)
    missing = int(np.maximum(want - held, 0).sum())
    surplus = int(np.maximum(held - want, 0).sum())
    spare = max(0, missing - surplus) // 2 if case["short"] else missing + 64
    rng = np.random.default_rng(int(seed))
    used = int(held.sum())
    perm = rng.permutation(used + spare).astype(np.int32)
    table = np.zeros((case["batch"], int(max(held.max(), want.max(), 1)) + 2), np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = perm[at:at + n]
        at += int(n)
    free = np.zeros(used + spare, np.int32)
    free[:spare] = perm[used:]
    return table, free, spare


def _theta(case):
    """Angle of each pair per position, in float64."""
    R = case["rdim"]
    return case["base"] ** (-2.0 * np.arange(R // 2, dtype=np.float64) / R)


def _mask_words(case, parents, rows):
    words = max(1, (max(len(p) for p in parents) + 31) // 32)
    bits = np.zeros((rows, 32 * words), bool)
    at = 0
    for p in parents:
        bits[at:at + len(p), :len(p)] = _seen(case, p)
        at += len(p)
    return np.packbits(bits, axis=1, bitorder="little").view(np.int32)


class _State:
    """What a program holds; gives its handles back when it goes."""

    def __init__(self):
        self.rotary = self.layout = None

    def __del__(self):
        if self.rotary is None and self.layout is None:
            return
        from paper_2606_03077_amd import libra
        if self.rotary is not None:
            libra.libra_rotary_destroy(self.rotary)
        if self.layout is not None:
            libra.libra_kv_layout_destroy(self.layout)


def _handle(case, dim):
    from paper_2606_03077_amd import libra
    pairing = {"half": libra.LIBRA_ROTARY_HALF, "interleaved": libra.LIBRA_ROTARY_INTERLEAVED}
    return libra.libra_rotary_create(head_dim=dim, rotary_dim=case["rdim"],
                                     pairing=pairing[case["layout"]], base=case["base"])


def _device(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a).astype(dtype)).cuda()


def _cache(s, gen, pool, hkv):
    s.k = _normal(gen, (pool * hkv * PAGE * DIM,))
    s.v = _normal(gen, (pool * hkv * PAGE * DIM,))
    s.pool, s.hkv = pool, hkv


def _append_inputs(case, seed, gen):
    """(k, v caches, qkv, q weight, k weight, slots, positions, pages in the pool)."""
    hq, hkv, padding = case["hq"], case["hkv"], case["padding"]
    token, position, used = _append_rows(case)
    pool = used + 3
    place = np.random.default_rng(int(seed)).permutation(pool)
    slots = np.full(case["rows"] + padding, -1, np.int64)
    slots[:case["rows"]] = place[token // PAGE] * PAGE + token % PAGE
    positions = np.zeros(case["rows"] + padding, np.int32)
    positions[:case["rows"]] = position
    k = _normal(gen, (pool * hkv * PAGE * DIM,))
    v = _normal(gen, (pool * hkv * PAGE * DIM,))
    # A layer's projections as one product leaves them: a row's queries, keys, values.
    qkv = _normal(gen, (case["rows"] + padding, hq + 2 * hkv, DIM))
    return k, v, qkv, _weight(gen, DIM, qkv.dtype), _weight(gen, DIM, qkv.dtype), slots, positions, pool


def _train_inputs(case, gen):
    hq, hkv, dim, rows, dtype = (case["hq"], case["hkv"], case["dim"], case["rows"],
                                 TYPES[case["type"]])
    qkv = _normal(gen, (rows, hq + 2 * hkv, dim), dtype)
    dy = _normal(gen, (rows, hq + hkv, dim), dtype)
    positions = np.random.default_rng(case["shape"]).integers(0, 20000) + np.arange(rows)
    return qkv, dy, _weight(gen, dim, dtype), _weight(gen, dim, dtype), positions


def prepare(case, seed):
    s = _State()
    gen = _generator(seed)
    s.case, s.op = case, case["op"]
    if s.op == "map":
        prior, new, held, depths = _map_sizes(case)
        table, free, spare = _free_stack(case, seed)
        s.prior, s.new, s.held = _device(prior), _device(new), _device(held)
        s.table, s.free, s.num_free = _device(table), _device(free), _device([spare])
        s.stride = table.shape[1]
        s.depths = _device(depths) if case["depths"] else None
        rows = len(depths)
        s.slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
        s.positions = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s.starts = torch.zeros(case["batch"] + 1, dtype=torch.int32, device="cuda")
        s.refused = torch.zeros(case["batch"], dtype=torch.int32, device="cuda")
        s.held_out = torch.zeros_like(s.held)
        s.num_out = torch.zeros_like(s.num_free)
        return s
    if s.op == "append":
        s.hq, s.hkv = case["hq"], case["hkv"]
        s.k, s.v, s.qkv, s.wq, s.wk, slots, positions, s.pool = _append_inputs(case, seed, gen)
        s.slots, s.positions = _device(slots, np.int64), _device(positions)
        s.theta = torch.from_numpy(_theta(case)).cuda()
        s.q_out = torch.zeros((len(slots), s.hq, DIM), dtype=torch.bfloat16, device="cuda")
        if own:
            from paper_2606_03077_amd import libra
            s.rotary = _handle(case, DIM)
            s.layout = libra.libra_kv_layout_create(s.k, s.v, s.pool, s.hkv)
        return s
    if s.op == "train":
        s.hq, s.hkv = case["hq"], case["hkv"]
        s.qkv, s.dy, s.wq, s.wk, positions = _train_inputs(case, gen)
        s.positions = _device(positions)
        s.theta = torch.from_numpy(_theta(case)).cuda()
        if own:
            from paper_2606_03077_amd import libra
            s.rotary = _handle(case, case["dim"])
            rows, dim, dtype = case["rows"], case["dim"], s.qkv.dtype
            new = lambda heads: torch.empty((rows, heads, dim), dtype=dtype, device="cuda")
            s.out = new(s.hq), new(s.hkv) if s.hkv else None
            s.grad = new(s.hq), new(s.hkv) if s.hkv else None
            s.dw = torch.empty((2, dim), dtype=torch.float32, device="cuda")
            s.ws = torch.empty(libra.libra_qk_norm_rotary_workspace_bytes(rows, s.hq, s.hkv, dim),
                               dtype=torch.uint8, device="cuda")
        return s
    if s.op == "accept":
        prior, counts, accepted = _accept_sizes(case)
        pool, table = _placement(_pages(prior + case["nodes"]), seed)
        _cache(s, gen, pool, case["hkv"])
        s.prior, s.counts, s.accepted = _device(prior), _device(counts), _device(accepted)
        s.table, s.stride = _device(table), table.shape[1]
        if own:
            from paper_2606_03077_amd import libra
            s.layout = libra.libra_kv_layout_create(s.k, s.v, pool, s.hkv)
        return s
    prior, nodes, parents = _tree_sizes(case)
    rows = int(nodes.sum()) + case["padding"]
    pool, table = _placement(_pages(prior + nodes), seed)
    _cache(s, gen, pool, case["hkv"])
    s.hq, s.nodes, s.lens, s.parents = case["hq"], nodes.tolist(), prior.tolist(), parents
    s.q = _normal(gen, (rows, s.hq, DIM))
    s.prior = _device(prior)
    s.starts = _device(np.concatenate([[0], np.cumsum(nodes)]))
    s.mask = _device(_mask_words(case, parents, rows)) if case["mask"] else None
    s.seen = [torch.from_numpy(_seen(case, p)).cuda() for p in parents]
    s.table, s.stride = _device(table), table.shape[1]
    s.out = torch.zeros((rows, s.hq, DIM), dtype=torch.bfloat16, device="cuda")
    s.lse = torch.zeros((rows, s.hq), dtype=torch.float32, device="cuda")
    if own:
        from paper_2606_03077_amd import libra
        s.layout = libra.libra_kv_layout_create(s.k, s.v, pool, s.hkv)
        s.ws = torch.empty(libra.libra_tree_attn_workspace_bytes(rows, case["batch"], s.hq, s.hkv),
                           dtype=torch.uint8, device="cuda")
    return s


# --- one pass --------------------------------------------------------------------------

def run(s):
    return (_LIBRARY if own else _PLAIN)[s.op](s)


def _library_map(s):
    from paper_2606_03077_amd import libra
    libra.libra_kv_map(s.prior, s.new, s.held, s.table, s.stride, s.free, s.num_free, s.depths,
                       s.slots, s.positions, s.starts, s.held_out, s.num_out, s.refused)
    return [s.table, s.held_out, s.free, s.num_out, s.slots, s.positions, s.starts, s.refused]


def _library_append(s):
    from paper_2606_03077_amd import libra
    q, k, v = s.qkv.split([s.hq, s.hkv, s.hkv], dim=1)
    libra.libra_kv_append_norm(s.layout, s.rotary, s.positions, s.slots, q if s.hq else None, k, v,
                               s.wq if s.hq else None, s.wk, EPS, s.q_out if s.hq else None)
    return [s.k, s.v, s.q_out]


def _library_train(s):
    from paper_2606_03077_amd import libra
    q, k, _ = s.qkv.split([s.hq, s.hkv, s.hkv], dim=1)
    dq, dk = s.dy.split([s.hq, s.hkv], dim=1)
    keys = s.hkv > 0
    k, dk, wk, dwk = (k, dk, s.wk, s.dw[1]) if keys else (None, None, None, None)
    libra.libra_qk_norm_rotary(s.rotary, q, k, s.wq, wk, EPS, s.positions, s.out[0], s.out[1])
    libra.libra_qk_norm_rotary_backward(s.rotary, dq, dk, q, k, s.wq, wk, EPS, s.positions,
                                        s.grad[0], s.grad[1], s.dw[0], dwk, s.ws)
    return [s.out[0], s.grad[0], s.dw[0]] + ([s.out[1], s.grad[1], s.dw[1]] if keys else [])


def _library_tree(s):
    from paper_2606_03077_amd import libra
    libra.libra_tree_attn(s.layout, s.q, s.prior, s.starts, s.mask, s.table, s.stride, s.hq, SCALE,
                          s.ws, s.out, s.lse)
    return [s.out, s.lse]


def _library_accept(s):
    from paper_2606_03077_amd import libra
    libra.libra_kv_accept(s.layout, s.prior, s.accepted, s.counts, s.table, s.stride)
    return [s.k, s.v]


_LIBRARY = {"map": _library_map, "append": _library_append, "train": _library_train,
            "tree": _library_tree, "accept": _library_accept}


def _plain_map(s):
    B, columns = s.table.shape
    capacity = s.free.numel()
    want = (s.prior.long() + s.new + PAGE - 1) // PAGE
    held = s.held.long()
    column = torch.arange(columns, device="cuda")[None]
    back = (column >= want[:, None]) & (column < held[:, None])
    rank = back.flatten().cumsum(0).view(B, columns) - 1
    # Entries that stay go to a place behind the stack.
    stack = torch.cat([s.free, s.free.new_zeros(1)])
    stack.scatter_(0, torch.where(back, s.num_free + rank, capacity).flatten(), s.table.flatten())
    top = s.num_free.long() + back.sum()
    need = (want - held).clamp(min=0)
    upto = need.cumsum(0)
    refused = (need > 0) & (upto > top)
    first = upto - need
    fresh = (column >= held[:, None]) & (column < want[:, None]) & ~refused[:, None]
    source = (top - 1 - (first[:, None] + column - held[:, None])).clamp(0, capacity - 1)
    s.table.copy_(torch.where(fresh, stack[source], s.table))
    s.free.copy_(stack[:capacity])
    s.held_out.copy_(torch.where(refused, held, want))
    s.num_out.copy_(top - torch.where(refused, 0, need).sum())
    s.refused.copy_(refused)
    ends = s.new.long().cumsum(0)
    s.starts[1:] = ends
    s.starts[0] = 0
    row = torch.arange(s.slots.numel(), device="cuda")
    seq = torch.searchsorted(ends, row, right=True).clamp(max=B - 1)
    live = row < ends[-1]
    index = s.prior[seq] + row - s.starts[seq]
    page = s.table[seq, (index // PAGE).clamp(0, columns - 1)].long()
    s.slots.copy_(torch.where(live & ~refused[seq], page * PAGE + index % PAGE, -1))
    position = index if s.depths is None else s.prior[seq] + s.depths
    s.positions.copy_(torch.where(live, position, 0))
    return [s.table, s.held_out, s.free, s.num_out, s.slots, s.positions, s.starts, s.refused]


def _turn(x, positions, theta, layout, back=False):
    """x [rows, heads, D] in float32, turned (back: by the negative angle)."""
    R = 2 * theta.numel()
    angle = positions.double()[:, None] * theta[None]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if back:
        sin = -sin
    out = x.clone()
    if layout == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        out[..., :R // 2] = a * cos - b * sin
        out[..., R // 2:R] = b * cos + a * sin
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        out[..., 0:R:2] = a * cos - b * sin
        out[..., 1:R:2] = b * cos + a * sin
    return out


def _norm_turn(s, x, weight, positions):
    f = x.float()
    r = (f.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
    return _turn(f * r * weight.float(), positions, s.theta, s.case["layout"]).to(x.dtype)


def _tiles(s):
    """Views of the cache: K [page, head, block, slot, 8], V [page, head, 2, channel, 2, 4]."""
    return (s.k.view(s.pool, s.hkv, 16, PAGE, 8), s.v.view(s.pool, s.hkv, 2, DIM, 2, 4))


def _plain_append(s):
    q, k, v = s.qkv.split([s.hq, s.hkv, s.hkv], dim=1)
    live = s.slots >= 0
    q, k, v, slots, positions = q[live], k[live], v[live], s.slots[live], s.positions[live]
    page, slot = slots // PAGE, slots % PAGE
    kt, vt = _tiles(s)
    kt[page, :, :, slot] = _norm_turn(s, k, s.wk, positions).reshape(-1, s.hkv, 16, 8)
    vt[page, :, slot // 4 % 2, :, slot // 8, slot % 4] = v
    s.q_out[live] = _norm_turn(s, q, s.wq, positions)
    return [s.k, s.v, s.q_out]


def _plain_train(s):
    q, k, _ = s.qkv.split([s.hq, s.hkv, s.hkv], dim=1)
    dq, dk = s.dy.split([s.hq, s.hkv], dim=1)
    out = []
    for x, dy, weight in ((q, dq, s.wq), (k, dk, s.wk)):
        if x.shape[1] == 0:
            continue
        f, w = x.float(), weight.float()
        r = (f.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
        n = f * r
        y = _turn(n * w, s.positions, s.theta, s.case["layout"]).to(x.dtype)
        du = _turn(dy.float(), s.positions, s.theta, s.case["layout"], back=True)
        dw = (du * n).sum(dim=(0, 1), dtype=torch.float64).float()
        dn = du * w
        dx = (r * (dn - n * (dn * n).mean(dim=-1, keepdim=True))).to(x.dtype)
        out += [y, dx, dw]
    return out


def _plain_tree(s):
    kt, vt = _tiles(s)
    G, row = s.hq // s.hkv, 0
    for b, (P, N) in enumerate(zip(s.lens, s.nodes)):
        ids = s.table[b, :(P + N + PAGE - 1) // PAGE].long()
        keys = kt[ids].permute(1, 0, 3, 2, 4).reshape(s.hkv, -1, DIM)[:, :P + N].float()
        vals = vt[ids].permute(1, 0, 4, 2, 5, 3).reshape(s.hkv, -1, DIM)[:, :P + N].float()
        qs = s.q[row:row + N].float().view(N, s.hkv, G, DIM).transpose(0, 1)
        z = torch.matmul(qs.reshape(s.hkv, -1, DIM), keys.transpose(1, 2)) * SCALE
        z = z.view(s.hkv, N, G, P + N)
        z[..., P:].masked_fill_(~s.seen[b][None, :, None], -math.inf)
        m = z.amax(dim=-1, keepdim=True)
        p = (z - m).exp()
        t = p.sum(dim=-1, keepdim=True)
        o = torch.matmul(p.view(s.hkv, -1, P + N), vals).view(s.hkv, N, G, DIM) / t
        s.out[row:row + N] = o.transpose(0, 1).reshape(N, s.hq, DIM)
        s.lse[row:row + N] = (m + t.log())[..., 0].transpose(0, 1).reshape(N, s.hq)
        row += N
    return [s.out, s.lse]


def _plain_accept(s):
    kt, vt = _tiles(s)
    at = torch.arange(s.accepted.shape[1], device="cuda")[None]
    live = at < s.counts[:, None]
    seq = torch.arange(s.accepted.shape[0], device="cuda")[:, None].expand_as(live)[live]
    to, of = (s.prior[:, None] + at)[live], (s.prior[:, None] + s.accepted)[live]
    pt, po = s.table[seq, to // PAGE].long(), s.table[seq, of // PAGE].long()
    st, so = to % PAGE, of % PAGE
    kt[pt, :, :, st] = kt[po, :, :, so]
    vt[pt, :, st // 4 % 2, :, st // 8, st % 4] = vt[po, :, so // 4 % 2, :, so // 8, so % 4]
    return [s.k, s.v]


_PLAIN = {"map": _plain_map, "append": _plain_append, "train": _plain_train, "tree": _plain_tree,
          "accept": _plain_accept}


# --- the same in float64 ---------------------------------------------------------------

def _exact_map(case, seed):
    """Request by request, as a host's allocator goes."""
    prior, new, held, depths = _map_sizes(case)
    table, free, spare = _free_stack(case, seed)
    rows = len(depths)
    stack = free[:spare].tolist()
    want = _pages(prior + new)
    for b in range(case["batch"]):
        stack += table[b, want[b]:held[b]].tolist()
    free[:len(stack)] = stack
    held_out, refused, asked, top = held.copy(), np.zeros(case["batch"], np.int64), 0, len(stack)
    slots, positions = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    starts = np.zeros(case["batch"] + 1, np.int64)
    for b in range(case["batch"]):
        asked += max(0, int(want[b] - held[b]))
        refused[b] = want[b] > held[b] and asked > top
        if not refused[b]:
            for j in range(int(held[b]), int(want[b])):
                table[b, j] = stack.pop()
            held_out[b] = want[b]
        starts[b + 1] = starts[b] + new[b]
        r = np.arange(starts[b], starts[b + 1])
        t = prior[b] + r - starts[b]
        positions[r] = prior[b] + depths[r] if case["depths"] else t
        if not refused[b]:
            slots[r] = table[b, t // PAGE].astype(np.int64) * PAGE + t % PAGE
    return [torch.from_numpy(np.asarray(x).astype(np.float64)).cuda()
            for x in (table, held_out, free, [len(stack)], slots, positions, starts, refused)]


def _turned64(x, positions, case, back=False):
    """One complex product per pair: (x1 + i x2) e^(i angle); x is float64."""
    R, D = case["rdim"], x.shape[-1]
    angle = torch.from_numpy(_theta(case)).to(x.device) * positions.double()[:, None]
    factor = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None, :]
    head, rest = x[..., :R], x[..., R:]
    if case["layout"] == "half":
        z = torch.complex(head[..., :R // 2].contiguous(), head[..., R // 2:].contiguous())
        z = z * factor
        turned = torch.cat([z.real, z.imag], dim=-1)
    else:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], R // 2, 2).contiguous()) * factor
        turned = torch.view_as_real(z).reshape(head.shape)
    return torch.cat([turned, rest], dim=-1) if R < D else turned


def _exact_append(case, seed):
    k, v, qkv, wq, wk, slots, positions, pool = _append_inputs(case, seed, _generator(seed))
    hq, hkv, rows = case["hq"], case["hkv"], case["rows"]
    at, p = torch.from_numpy(slots[:rows]).cuda(), torch.from_numpy(positions[:rows]).cuda()
    page, slot = at // PAGE, at % PAGE
    weight = torch.cat([wq.double().expand(hq, DIM), wk.double().expand(hkv, DIM)])
    turned = []
    for r in range(0, rows, 4096):
        x = qkv[r:min(rows, r + 4096), :hq + hkv].double()
        size = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
        n = x / torch.sqrt(size * size / DIM + EPS)
        turned.append(_turned64(n * weight, p[r:r + 4096], case))
    turned = torch.cat(turned)
    d = torch.arange(DIM, device="cuda")
    k64, v64 = k.double(), v.double()
    for g in range(hkv):  # element addresses of the new tokens in the flat caches
        tile = (page * hkv + g) * (PAGE * DIM)
        k64[tile[:, None] + (d // 8 * PAGE)[None] * 8 + slot[:, None] * 8 + d % 8] = \
            turned[:, hq + g]
        v64[tile[:, None] + ((slot // 4 % 2) * DIM)[:, None] * 8 + d * 8
            + (slot // 8 * 4 + slot % 4)[:, None]] = qkv[:rows, hq + hkv + g].double()
    q = torch.zeros((len(slots), hq, DIM), dtype=torch.float64, device="cuda")
    q[:rows] = turned[:, :hq]
    return [k64, v64, q]


def _exact_train(case, seed):
    """The forward pass as an expression, its gradients through it."""
    qkv, dy, wq, wk, positions = _train_inputs(case, _generator(seed))
    hq, hkv, rows = case["hq"], case["hkv"], case["rows"]
    p = torch.from_numpy(positions).cuda()
    out = []
    for h0, h1, weight in ((0, hq, wq), (hq, hq + hkv, wk)):
        if h0 == h1:
            continue
        w = weight.double().requires_grad_()
        ys, dxs = [], []
        for r in range(0, rows, 2048):
            x = qkv[r:min(rows, r + 2048), h0:h1].double().requires_grad_()
            n = x / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / x.shape[-1] + EPS)
            y = _turned64(n * w, p[r:r + 2048], case)
            y.backward(dy[r:r + 2048, h0:h1].double())
            ys.append(y.detach())
            dxs.append(x.grad)
        out += [torch.cat(ys), torch.cat(dxs), w.grad]
    return out


def _exact_tree(case, seed):
    gen = _generator(seed)
    hq, hkv = case["hq"], case["hkv"]
    prior, nodes, parents = _tree_sizes(case)
    rows = int(nodes.sum()) + case["padding"]
    pool, table = _placement(_pages(prior + nodes), seed)
    k = _normal(gen, (pool * hkv * PAGE * DIM,))
    v = _normal(gen, (pool * hkv * PAGE * DIM,))
    q = _normal(gen, (rows, hq, DIM))
    out = torch.zeros((rows, hq, DIM), dtype=torch.float64, device="cuda")
    lse = torch.zeros((rows, hq), dtype=torch.float64, device="cuda")
    d = torch.arange(DIM, device="cuda")
    G, r0 = hq // hkv, 0
    for b in range(case["batch"]):
        P, N = int(prior[b]), int(nodes[b])
        t = torch.arange(P + N, device="cuda")
        ids = torch.from_numpy(table[b].astype(np.int64)).cuda()[t // PAGE]
        sl = t % PAGE
        unseen = torch.zeros((N, P + N), dtype=torch.bool, device="cuda")
        unseen[:, P:] = ~torch.from_numpy(_seen(case, parents[b])).cuda()
        unseen = unseen.repeat_interleave(G, dim=0)
        for g in range(hkv):
            tile = ((ids * hkv + g) * (PAGE * DIM))[:, None]
            K = k[tile + (d // 8 * PAGE * 8 + d % 8)[None] + (sl * 8)[:, None]].double()
            V = v[tile + (d * 8)[None]
                  + (sl // 4 % 2 * DIM * 8 + sl // 8 * 4 + sl % 4)[:, None]].double()
            z = q[r0:r0 + N, g * G:(g + 1) * G].double().reshape(-1, DIM) @ K.t()
            z *= SCALE
            z[unseen] = -math.inf
            total = torch.logsumexp(z, dim=1)
            o = torch.exp(z - total[:, None]) @ V
            out[r0:r0 + N, g * G:(g + 1) * G] = o.view(N, G, DIM)
            lse[r0:r0 + N, g * G:(g + 1) * G] = total.view(N, G)
        r0 += N
    return [out, lse]


def _exact_accept(case, seed):
    """Element by element of the logical cache: token, head, channel."""
    gen = _generator(seed)
    hkv = case["hkv"]
    prior, counts, accepted = _accept_sizes(case)
    pool, table = _placement(_pages(prior + case["nodes"]), seed)
    k = _normal(gen, (pool * hkv * PAGE * DIM,))
    v = _normal(gen, (pool * hkv * PAGE * DIM,))
    to, of = [], []
    for b in range(case["batch"]):
        for i in range(int(counts[b])):
            for where, token in ((to, int(prior[b]) + i), (of, int(prior[b] + accepted[b, i]))):
                where.append(int(table[b, token // PAGE]) * PAGE + token % PAGE)
    to, of = (torch.tensor(x, device="cuda")[:, None, None] for x in (to, of))
    g, d = torch.arange(hkv, device="cuda")[None, :, None], torch.arange(DIM, device="cuda")
    at_k = lambda s: (s // PAGE * hkv + g) * PAGE * DIM + (d // 8 * PAGE + s % PAGE) * 8 + d % 8
    at_v = lambda s: ((s // PAGE * hkv + g) * PAGE * DIM + (s // 4 % 2 * DIM + d) * 8
                      + s % PAGE // 8 * 4 + s % 4)
    k64, v64 = k.double(), v.double()
    k64[at_k(to)] = k[at_k(of)].double()
    v64[at_v(to)] = v[at_v(of)].double()
    return [k64, v64]


_EXACT = {"map": _exact_map, "append": _exact_append, "train": _exact_train, "tree": _exact_tree,
          "accept": _exact_accept}


def exact(case, seed):
    return _EXACT[case["op"]](case, seed)
