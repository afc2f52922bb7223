"""The forms that only large calls of libra_rotary_apply and libra_kv_append take: four heads to a
thread, reads and writes past the caches, several launches.

Every form gives the same bits, so a large call is compared with small ones (whose results
test_gpu_rotary.py holds against float64), and some of its rows with float64 directly."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra

import gpu_harness as H
from test_gpu_kv_append import Cache, check_cache
from test_gpu_rotary import Handle, f64, positions_of, randn

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
SMALL = 256                 # rows of a call that takes one head to a thread: 50 heads of 256 are 409,600 pieces


def bits(t):
    return t.view(torch.int32 if t.dtype is FP32 else torch.int16)


def by_small_calls(rope, x, pd, backward):
    out = torch.empty(x.shape, dtype=x.dtype, device="cuda")
    for r in range(0, x.shape[0], SMALL):
        part = x[r:r + SMALL].contiguous()
        libra.libra_rotary_apply(rope.h, part, pd[r:r + SMALL], out[r:r + SMALL], backward=backward)
    return out


# Four heads to a thread from 40,960 vectors of 128 channels on; 1,100 rows of 40 heads read past
# the caches where an instruction covers whole lines, and 128 MiB are written past them too.
ROWS = [(1100, 40, 128, 64, False, BF16), (1100, 40, 128, 96, False, FP16), (1100, 40, 128, 128, False, BF16),
        (1100, 40, 128, 64, True, BF16), (1100, 41, 128, 32, True, FP16), (1100, 40, 128, 64, False, FP32),
        (1100, 40, 128, 48, True, FP32), (5000, 17, 72, 24, False, BF16), (1030, 64, 80, 80, True, FP16),
        (13200, 40, 128, 128, False, BF16), (13200, 40, 128, 128, False, FP16),
        (13200, 40, 128, 64, True, BF16), (7001, 40, 128, 64, False, FP32), (6000, 50, 256, 128, True, BF16)]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("rows,heads,dim,rdim,interleaved,dtype", ROWS)
def test_large_rows(rows, heads, dim, rdim, interleaved, dtype, backward):
    H.say(f"[case] large rows {rows}x{heads}x{dim} R={rdim} inter={interleaved} {dtype} backward={backward}")
    rope = Handle(dim, rdim, interleaved, amplitude=1.25)
    buf = randn((rows, heads + 3, dim), dtype, 1)
    x = buf[:, 1:1 + heads]
    p, pd = positions_of(rows, 2)
    out = torch.full((rows + 1, heads, dim), 5.0, dtype=dtype, device="cuda")
    libra.libra_rotary_apply(rope.h, x, pd, out[:rows], backward=backward)
    torch.cuda.synchronize()
    want = by_small_calls(rope, x, pd, backward)
    assert torch.equal(bits(out[:rows]), bits(want)) and bool((out[rows] == 5.0).all())
    look = torch.tensor(sorted({0, 1, rows // 3, rows // 2 + 1, rows - 2, rows - 1}), device="cuda")
    rope.check(f64(out[look]), f64(x[look]), p[look.cpu().numpy()], dtype, backward, "rows")
    rest = buf[:, [0, heads + 1, heads + 2]].clone()
    libra.libra_rotary_apply(rope.h, x, pd, x, backward=backward)
    assert torch.equal(bits(x.contiguous()), bits(want)), "in place"
    assert torch.equal(bits(buf[:, [0, heads + 1, heads + 2]].contiguous()), bits(rest)), "beside x"
    rope.close()


def chunk_slots(rows, pages, rng):
    """Chunks that begin anywhere in a page, single rows and padding, in slots of their own."""
    perm, out, page = rng.permutation(pages), [], 0
    while len(out) < rows:
        n = int(rng.choice([1, 1, 17, 130, 900]))
        first = int(rng.integers(16))
        out += [int(perm[page + (first + i) // 16]) * 16 + (first + i) % 16 for i in range(n)]
        page += (first + n + 15) // 16
        out += [-1] * int(rng.choice([0, 0, 1, 20]))
    return np.array(out[:rows], np.int64)


@pytest.mark.parametrize("rows", [1100, 9500])          # through the caches, and past them
@pytest.mark.parametrize("kw", [dict(), dict(rdim=64), dict(interleaved=True), dict(rdim=64, interleaved=True),
                                dict(rdim=96, amplitude=1.25), dict(rdim=20), dict(rdim=22, interleaved=True)],
                         ids=str)
def test_large_append(kw, rows):
    hq, hkv, pages = 40, 8, 3 * rows // 16 + 200
    H.say(f"[case] large append {rows} rows {kw}")
    rng = np.random.default_rng(rows)
    cache, rope = Cache(pages, hkv), Handle(**kw)
    slots = chunk_slots(rows, pages, rng)
    live = torch.from_numpy(slots >= 0).cuda()
    pos = rng.integers(0, 200000, size=rows).astype(np.int32)
    pd, sd = torch.from_numpy(pos).cuda(), torch.from_numpy(slots).cuda()
    qkv = randn((rows, hq + 2 * hkv, 128), BF16, 3)
    q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    q_out = torch.full((rows + 1, hq, 128), 5.0, dtype=BF16, device="cuda")
    libra.libra_kv_append(cache.layout, rope.h, pd, sd, q, k, v, q_out[:rows])
    torch.cuda.synchronize()
    want_q, want_k = (by_small_calls(rope, t, pd, False) for t in (q, k))
    assert torch.equal(q_out[:rows][live], want_q[live])
    assert bool((q_out[:rows][~live] == 5.0).all()) and bool((q_out[rows] == 5.0).all())
    at, (gk, gv), (k0, v0) = sd[live], cache.logical(), cache.initial()
    k0[at], v0[at] = want_k[live], v[live]
    assert torch.equal(gk, k0) and torch.equal(gv, v0)
    dense = q.contiguous()
    libra.libra_kv_append(cache.layout, rope.h, pd, sd, dense, k, v, dense)
    assert torch.equal(dense, torch.where(live[:, None, None], want_q, q)), "in place"
    rope.close()
    cache.close()


# One launch takes 2^22 blocks of queries: of a row of 15 heads, or of 16 rows of a head.
@pytest.mark.parametrize("kw,hq,per_launch", [(dict(rdim=64), 15, 2 ** 22),
                                              (dict(rdim=20), 65535, 2 ** 22 // 65535 * 16)], ids=str)
def test_append_with_queries_in_several_launches(kw, hq, per_launch):
    """17 GB of queries; only the rows around the second launch's first are not padding."""
    H.say(f"[case] append in several launches {kw} hq={hq}")
    rows, first, n = per_launch + 50, per_launch - 21, 60
    cache, rope = Cache(8, 1), Handle(**kw)
    q = torch.zeros((rows, hq, 128), dtype=BF16, device="cuda")
    k, v = (torch.zeros((rows, 1, 128), dtype=BF16, device="cuda") for _ in range(2))
    near = slice(first - 30, rows)
    q[near], k[near], v[near] = (randn((rows - first + 30, h, 128), BF16, s) for s, h in ((5, hq), (6, 1), (7, 1)))
    slots = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    slots[first:first + n] = torch.arange(5, 5 + n, device="cuda")
    pd = torch.arange(rows, dtype=torch.int32, device="cuda")
    before = q[near].clone()
    libra.libra_kv_append(cache.layout, rope.h, pd, slots, q, k, v, q)
    torch.cuda.synchronize()
    live = slice(first, first + n)
    check_cache(cache, rope, slots[live].cpu().numpy(), pd[live].cpu().numpy(), k[live], v[live], "launches")
    want = before.clone()
    libra.libra_rotary_apply(rope.h, before[30:30 + n].contiguous(), pd[live], want[30:30 + n])
    assert torch.equal(q[near], want)
    assert not bool(q[:first - 30].any())
    rope.close()
    cache.close()
