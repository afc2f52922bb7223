"""Norms of heads with rotary positions on the GPU: forward, gradients and the cache append, against
the float64 oracle.

Tolerances, per element.  A head's sum of squares adds at most D / lanes + 6 float32 products in
a row; with the square root and the two products that is c = (D / 8 + 12) 2^-24 of the value, and of
every term of a turned pair; cosine and sine are within 1.2e-7 of theirs.  The result is rounded
once: eps / 2 of its type.  Gradients add the mean (c again) and three products.  Weight gradients
add float32 terms in chains: at most the rows and heads that a thread takes, and the workgroup's
threads' after."""
import numpy as np
import pytest
import torch

from oracle import drafts as ref
from oracle import rotary
from paper_2606_03077_amd import libra

from test_gpu_kv_append import Cache, runs

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


class Handle:
    def __init__(self, dim=128, rdim=0, interleaved=False, amplitude=1.0, base=1e4):
        self.h = libra.libra_rotary_create(head_dim=dim, rotary_dim=rdim, base=base, amplitude=amplitude,
                                           pairing=int(interleaved))
        self.theta = rotary.frequencies(rdim or dim, base)
        self.turn = dict(interleaved=interleaved, amplitude=amplitude)

    def __del__(self):
        libra.libra_rotary_destroy(self.h)


def f64(t):
    return t.double().cpu().numpy()


def randn(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def weights(dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.2 * torch.randn(dim, generator=g)).to(dtype).cuda()


def rounding(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, tol, what):
    got = f64(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.2f} tol"


def check_forward(x, w, hd, pos, y, what, eps=EPS):
    want, n, r = ref.norm_turn(f64(x), f64(w), eps, pos, hd.theta, **hd.turn)
    u = n * f64(w)
    size = rotary.partner_size(u, hd.theta, hd.turn["interleaved"])
    size = np.where(size > 0, size, np.abs(u)) * hd.turn["amplitude"]
    D = x.shape[-1]
    tiny = 2.0 ** -24 if x.dtype == torch.float16 else 1e-38  # half the least step of small fp16 numbers
    close(y, want, ((D / 8 + 12) * 2.0 ** -24 + 1.3e-7) * size + rounding(x.dtype) * np.abs(want) * 1.01 + tiny, what)


def check_backward(x, w, dy, hd, pos, dx, dw, what, eps=EPS):
    want, want_w, (size, size_w) = ref.norm_turn_grad(f64(x), f64(w), eps, pos, hd.theta, f64(dy), **hd.turn)
    D, count = x.shape[-1], x.shape[0] * x.shape[1]
    c = (D / 8 + 16) * 2.0 ** -24 + 1.3e-7
    tiny = 2.0 ** -24 if x.dtype == torch.float16 else 1e-38
    close(dx, want, 3 * c * size + rounding(x.dtype) * np.abs(want) * 1.01 + tiny, what + " dx")
    if dw is not None:
        close(dw, want_w, (c + (min(count, 4096) + 40) * 2.0 ** -24) * size_w + 2.0 ** -24 * np.abs(want_w), what + " dw")


def run_forward(hd, q, k, wq, wk, pos, qo=None, ko=None, eps=EPS):
    qo = torch.full_like(q, float("nan")) if qo is None and q is not None else qo
    ko = torch.full_like(k, float("nan")) if ko is None and k is not None else ko
    libra.libra_qk_norm_rotary(hd.h, q, k, wq, wk, eps, torch.from_numpy(pos).int().cuda(), qo, ko)
    torch.cuda.synchronize()
    return qo, ko


def run_backward(hd, q, k, wq, wk, pos, gq, gk, dq=None, dk=None, weight_grads=True, eps=EPS):
    x = q if q is not None else k
    D = x.shape[2]
    dq = torch.full_like(q, float("nan")) if dq is None and q is not None else dq
    dk = torch.full_like(k, float("nan")) if dk is None and k is not None else dk
    dw = torch.full((2, D), float("nan"), device="cuda") if weight_grads else (None, None)
    ws = torch.full((libra.libra_qk_norm_rotary_workspace_bytes(*x.shape[:2], 0, D),), 255,
                    dtype=torch.uint8, device="cuda") if weight_grads else None
    libra.libra_qk_norm_rotary_backward(hd.h, gq, gk, q, k, wq, wk, eps, torch.from_numpy(pos).int().cuda(),
                                        dq, dk, dw[0] if q is not None else None,
                                        dw[1] if k is not None else None, ws)
    torch.cuda.synchronize()
    return dq, dk, dw[0], dw[1]


ROPES = [dict(), dict(rdim=64, interleaved=True), dict(rdim=20), dict(rdim=96, amplitude=1.25),
         dict(rdim=22, interleaved=True), dict(rdim=2)]
SHAPES = [(1, 1, 1), (1, 28, 4), (3, 5, 2), (17, 40, 8), (130, 7, 1), (33, 64, 0), (2000, 16, 4)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rope", ROPES, ids=str)
@pytest.mark.parametrize("rows,hq,hk", SHAPES)
def test_forward_and_gradients(dtype, rope, rows, hq, hk):
    hd, t = Handle(**rope), TYPES[dtype]
    qkv = randn((rows, hq + 2 * hk + 1, 128), t, rows + hq)  # slices of one projection
    q, k = qkv[:, :hq], qkv[:, hq:hq + hk] if hk else None
    wq, wk = weights(128, t, 1), weights(128, t, 2) if hk else None
    pos = np.random.default_rng(rows).integers(-5, 100000, size=rows)
    qo, ko = run_forward(hd, q, k, wq, wk, pos)
    check_forward(q, wq, hd, pos, qo, "q")
    gq, gk = randn((rows, hq, 128), t, 7), randn((rows, hk, 128), t, 8) if hk else None
    dq, dk, dwq, dwk = run_backward(hd, q, k, wq, wk, pos, gq, gk)
    check_backward(q, wq, gq, hd, pos, dq, dwq, "q")
    if hk:
        check_forward(k, wk, hd, pos, ko, "k")
        check_backward(k, wk, gk, hd, pos, dk, dwk, "k")
        # Alone, either gives the same bits.
        alone, _ = run_forward(hd, k, None, wk, None, pos)
        assert torch.equal(alone, ko)
        _, alone = run_forward(hd, None, k, None, wk, pos)
        assert torch.equal(alone, ko)


@pytest.mark.parametrize("dim,rdim", [(2, 2), (6, 4), (8, 8), (16, 8), (64, 64), (64, 32), (80, 80), (100, 36),
                                      (256, 256), (256, 128), (512, 256), (500, 30)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_sizes(dim, rdim, dtype, interleaved):
    hd, t, rows = Handle(dim, rdim, interleaved), TYPES[dtype], 37
    q, k = randn((rows, 5, dim), t, 1), randn((rows, 2, dim), t, 2)
    wq, wk = weights(dim, torch.float32, 3), weights(dim, torch.float32, 4)
    pos = np.arange(rows) * 31
    for x, w, y in zip((q, k), (wq, wk), run_forward(hd, q, k, wq, wk, pos)):
        check_forward(x, w, hd, pos, y, "y")
    gq, gk = randn(q.shape, t, 5), randn(k.shape, t, 6)
    dq, dk, dwq, dwk = run_backward(hd, q, k, wq, wk, pos, gq, gk)
    check_backward(q, wq, gq, hd, pos, dq, dwq, "q")
    check_backward(k, wk, gk, hd, pos, dk, dwk, "k")


@pytest.mark.parametrize("wtype", list(TYPES))
@pytest.mark.parametrize("layout", ["heads first", "odd rows", "unaligned", "broadcast"])
def test_layouts_and_weight_types(wtype, layout):
    hd, rows, heads = Handle(), 19, 6
    base = randn((rows * heads * 140 + 64,), torch.bfloat16, 1)
    strided = lambda row, head, off: base.as_strided((rows, heads, 128), (row, head, 1), off)
    x = {"heads first": strided(128, 128 * rows, 0), "odd rows": strided(heads * 128 + 3, 128, 0),
         "unaligned": strided(heads * 128, 128, 1), "broadcast": strided(128, 0, 0)}[layout]
    w = weights(128, TYPES[wtype], 2)
    pos = np.arange(rows) + 5
    out = torch.full((heads, rows, 128), float("nan"), dtype=x.dtype, device="cuda").transpose(0, 1)
    y, _ = run_forward(hd, x, None, w, None, pos, out)
    check_forward(x, w, hd, pos, y, layout)
    dy = randn((1, 1, 128), torch.bfloat16, 9).expand(rows, heads, 128)  # a broadcast gradient
    dx, _, dw, _ = run_backward(hd, x, None, w, None, pos, dy, None, torch.full_like(out, 0.0))
    check_backward(x, w, dy, hd, pos, dx, dw, layout)


@pytest.mark.parametrize("rope", [dict(), dict(rdim=20)], ids=str)
def test_in_place(rope):
    hd, rows = Handle(**rope), 70
    q, k = randn((rows, 9, 128), torch.bfloat16, 1), randn((rows, 3, 128), torch.bfloat16, 2)
    w, pos = weights(128, torch.bfloat16, 3), np.arange(rows)
    qo, ko = run_forward(hd, q, k, w, w, pos)
    gq, gk = randn(q.shape, q.dtype, 4), randn(k.shape, k.dtype, 5)
    dq, dk, dwq, dwk = run_backward(hd, q, k, w, w, pos, gq, gk)
    for into in ("x", "grad"):
        a = [t.clone() for t in (q, k, gq, gk)]
        out = a[:2] if into == "x" else a[2:]
        eq, ek, ewq, ewk = run_backward(hd, a[0], a[1], w, w, pos, a[2], a[3], *out)
        assert all(torch.equal(x, y) for x, y in ((dq, eq), (dk, ek), (dwq, ewq), (dwk, ewk)))
    run_forward(hd, q, k, w, w, pos, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_no_rows_and_no_weight_gradients():
    hd = Handle()
    x, w = torch.empty((0, 3, 128), dtype=torch.bfloat16, device="cuda"), weights(128, torch.bfloat16, 1)
    _, _, dwq, dwk = run_backward(hd, x, x, w, w, np.arange(0), x, x)
    assert (dwq == 0).all() and (dwk == 0).all()
    x, g = randn((40, 3, 128), torch.bfloat16, 1), randn((40, 3, 128), torch.bfloat16, 2)
    full = run_backward(hd, x, None, w, None, np.arange(40), g, None)
    dx, _, _, _ = run_backward(hd, x, None, w, None, np.arange(40), g, None, weight_grads=False)
    assert torch.equal(dx, full[0])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_small_zero_large_and_nonfinite_heads(dtype):
    t = TYPES[dtype]
    hd, eps = Handle(), 1e-5
    x, w = randn((8, 2, 128), t, 1), weights(128, t, 2)
    x[0], x[1, 0], x[2, 0] = 0, x[1, 0] * 1e-4, x[2, 0] * 100
    g = randn(x.shape, t, 3)
    pos = np.arange(8)
    y, _ = run_forward(hd, x, None, w, None, pos, eps=eps)
    check_forward(x, w, hd, pos, y, "y", eps)
    dx, _, dw, _ = run_backward(hd, x, None, w, None, pos, g, None, eps=eps)
    check_backward(x, w, g, hd, pos, dx, dw, "dx", eps)
    assert (y[0] == 0).all()
    x[3, 1, 5], x[4, 0, 7] = float("nan"), float("inf")
    z, _ = run_forward(hd, x, None, w, None, pos, eps=eps)
    assert z[3, 1].isnan().all()
    other = torch.ones(8, 2, dtype=torch.bool)
    other[3, 1] = other[4, 0] = False
    assert torch.equal(z[other.cuda()], y[other.cuda()])


def test_many_rows_and_replayed_gradients():
    """Rows past one workgroup's, and a captured training pass beside its eager one."""
    hd, rows = Handle(rdim=64, interleaved=True), 5000
    qkv = randn((rows, 12, 128), torch.float32, 1)
    q, k = qkv[:, :8], qkv[:, 8:10]
    wq, wk = weights(128, torch.bfloat16, 2), weights(128, torch.bfloat16, 3)
    pos = np.arange(rows)
    gq, gk = randn(q.shape, q.dtype, 4), randn(k.shape, k.dtype, 5)
    eager = run_forward(hd, q, k, wq, wk, pos) + run_backward(hd, q, k, wq, wk, pos, gq, gk)
    check_backward(q, wq, gq, hd, pos, eager[2], eager[4], "q")
    p = torch.from_numpy(pos).int().cuda()
    outs = [torch.zeros_like(t) for t in eager]
    ws = torch.zeros(libra.libra_qk_norm_rotary_workspace_bytes(rows, 8, 2, 128), dtype=torch.uint8,
                     device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        libra.libra_qk_norm_rotary(hd.h, q, k, wq, wk, EPS, p, outs[0], outs[1])
        libra.libra_qk_norm_rotary_backward(hd.h, gq, gk, q, k, wq, wk, EPS, p, *outs[2:], ws)
    for _ in range(3):
        for t in outs:
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


@pytest.mark.parametrize("dtype,rows", [("bf16", 10007), ("fp32", 5003)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_past_the_caches(dtype, rows, interleaved):
    """Beyond the size from which the gradient goes past the caches: the bits of a part of the rows."""
    hd, t, pos = Handle(rdim=64, interleaved=interleaved), TYPES[dtype], np.arange(rows)
    q, k = randn((rows, 12, 128), t, 1), randn((rows, 2, 128), t, 2)
    gq, gk = randn(q.shape, t, 3), randn(k.shape, t, 4)
    wq, wk = weights(128, t, 5), weights(128, t, 6)
    dq, dk, _, dwk = run_backward(hd, q, k, wq, wk, pos, gq, gk)
    check_backward(k, wk, gk, hd, pos, dk, dwk, "k")
    at = slice(rows - 300, rows)
    few = run_backward(hd, q[at], k[at], wq, wk, pos[at], gq[at], gk[at])
    assert torch.equal(few[0], dq[at]) and torch.equal(few[1], dk[at])


def test_on_another_stream():
    hd, rows, s = Handle(), 300, torch.cuda.Stream()
    q, g, w, pos = randn((rows, 4, 128), torch.bfloat16, 1), randn((rows, 4, 128), torch.bfloat16, 2), \
        weights(128, torch.bfloat16, 3), np.arange(rows)
    want = run_forward(hd, q, None, w, None, pos)[0], *run_backward(hd, q, None, w, None, pos, g, None)[::2]
    y, dx, dw = torch.empty_like(q), torch.empty_like(q), torch.empty(128, device="cuda")
    ws = torch.empty(libra.libra_qk_norm_rotary_workspace_bytes(rows, 4, 0, 128), dtype=torch.uint8, device="cuda")
    p = torch.from_numpy(pos).int().cuda()
    torch.cuda.synchronize()
    libra.libra_qk_norm_rotary(hd.h, q, None, w, None, EPS, p, y, None, stream=s)
    libra.libra_qk_norm_rotary_backward(hd.h, g, None, q, None, w, None, EPS, p, dx, None, dw, None, ws, stream=s)
    s.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and torch.equal(dw, want[2])


# --- the cache append ------------------------------------------------------------------------

@pytest.mark.parametrize("rope", ROPES, ids=str)
@pytest.mark.parametrize("pattern", ["one", "singles", "middle", "padded", "all_padding", "mixed"])
@pytest.mark.parametrize("hq,hkv", [(28, 4), (0, 1), (8, 8)])
def test_append(rope, pattern, hq, hkv):
    hd, pages = Handle(**rope), 60
    cache = Cache(pages, hkv)
    slots = np.array(runs(pattern, np.random.default_rng(5), pages), np.int64)
    rows = len(slots)
    qkv = randn((rows, hq + 2 * hkv, 128), torch.bfloat16, 1)
    q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    q = q if hq else None
    wq, wk = weights(128, torch.bfloat16, 2), weights(128, torch.bfloat16, 3)
    pos = np.random.default_rng(2).integers(0, 50000, size=rows)
    q_out = torch.full((rows, hq, 128), 7.0, dtype=torch.bfloat16, device="cuda") if hq else None
    libra.libra_kv_append_norm(cache.layout, hd.h, torch.from_numpy(pos).int().cuda(),
                               torch.from_numpy(slots).cuda(), q, k, v, wq if hq else None, wk, EPS, q_out)
    qo, ko = run_forward(hd, q, k, wq if hq else None, wk, pos)
    live = (slots >= 0) & (slots < pages * 16)
    want = cache.initial()
    at, lv = torch.from_numpy(slots[live]).cuda(), torch.from_numpy(live).cuda()
    want[0][at], want[1][at] = ko[lv], v[lv]
    for got, w in zip(cache.logical(), want):
        assert torch.equal(got, w)
    if hq:
        assert torch.equal(q_out[lv], qo[lv]) and (q_out[~lv] == 7.0).all()
    if live.any():
        check_forward(k[lv], wk, hd, pos[live], ko[lv], "k")
    cache.close()


def test_append_in_place_and_float32_weights():
    hd, cache = Handle(), Cache(20, 2)
    rows = 200
    q, kv = randn((rows, 6, 128), torch.bfloat16, 1), randn((rows, 4, 128), torch.bfloat16, 2)
    w = weights(128, torch.float32, 3)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    want, _ = run_forward(hd, q, None, w, None, np.arange(rows))
    libra.libra_kv_append_norm(cache.layout, hd.h, pos, pos.long() + 3, q, kv[:, :2], kv[:, 2:], w, w, EPS, q)
    torch.cuda.synchronize()
    assert torch.equal(q, want)
    cache.close()


def test_append_of_many_rows_streams():
    """Beyond the size from which queries go past the caches."""
    hd, hq, hkv, rows = Handle(base=1e6), 40, 8, 9600
    cache = Cache(rows // 16 + 1, hkv)
    qkv = randn((rows, hq + 2 * hkv, 128), torch.bfloat16, 1)
    q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    w = weights(128, torch.bfloat16, 3)
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    q_out = torch.empty((rows, hq, 128), dtype=torch.bfloat16, device="cuda")
    libra.libra_kv_append_norm(cache.layout, hd.h, pos, pos.long(), q, k, v, w, w, EPS, q_out)
    qo, ko = run_forward(hd, q, k, w, w, np.arange(rows))
    got = cache.logical()
    assert torch.equal(q_out, qo) and torch.equal(got[0][:rows], ko) and torch.equal(got[1][:rows], v)
    part = slice(rows - 50, rows)
    check_forward(q[part], w, hd, np.arange(rows)[part], qo[part], "q")
    cache.close()
