"""libra_rotary_apply on the GPU against the float64 oracle.

Tolerance, derived: cosine and sine are within 1.2e-7 of the exact ones (their angle within
1.5 * 2^-24 of at most pi / 4, the polynomial's roundings 2^-25 and less, the truncated turn
1.5e-9), the amplitude and the product round by 2^-24 each and the sum's rounding is the
output's in float32.  So |y - exact| <= A (|x1| + |x2|) (1.2e-7 + 2 * 6e-8), within 3e-7 of the
pair's size, and then half a step of the output's type.
"""
import numpy as np
import pytest
import torch

from oracle import rotary as ref
from paper_2606_03077_amd import libra

import gpu_harness as H

pytestmark = pytest.mark.gpu

ERR = 3e-7
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25, torch.float32: 1e-38}
SCALINGS = {"plain": libra.LIBRA_ROTARY_PLAIN, "linear": libra.LIBRA_ROTARY_LINEAR,
            "base": libra.LIBRA_ROTARY_BASE, "bands": libra.LIBRA_ROTARY_BANDS}


class Handle:
    """A rotary handle and the oracle's frequencies for it."""

    def __init__(self, dim=128, rdim=None, interleaved=False, amplitude=1.0, **kw):
        self.dim, self.rdim = dim, rdim or dim
        self.interleaved, self.amplitude = interleaved, amplitude
        self.theta = ref.frequencies(self.rdim, **kw)
        self.h = libra.libra_rotary_create(
            head_dim=dim, rotary_dim=self.rdim, pairing=int(interleaved), amplitude=amplitude,
            **dict(kw, scaling=SCALINGS[kw.get("scaling", "plain")]))

    def close(self):
        libra.libra_rotary_destroy(self.h)

    def turn(self, x, positions, backward=False):
        return ref.turn(x, positions, self.theta, self.interleaved, self.amplitude, backward)

    def check(self, got, x, positions, dtype, backward=False, label=""):
        """got and x: float64 [rows, heads, D]."""
        want = self.turn(x, positions, backward)
        slack = ERR * self.amplitude * ref.partner_size(x, self.theta, self.interleaved)
        turned = slack > 0
        tol = np.where(turned, slack + HALF_STEP[dtype] * (np.abs(want) + slack) + TINY[dtype], 0)
        worst = float((np.abs(got - want) - tol).max()) if got.size else 0.0
        H.say(f"[rotary] {label}: largest excess over the tolerance {worst:.2e}")
        assert (np.abs(got - want) <= tol).all(), label


def f64(t):
    return t.double().cpu().numpy()


def randn(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, dtype=dtype, device="cuda", generator=g)


def positions_of(rows, seed, lo=0, hi=40960):
    p = np.random.default_rng(seed).integers(lo, hi, size=rows).astype(np.int32)
    return p, torch.from_numpy(p).cuda()


SHAPES = [  # rows, heads, dim, rotary_dim
    (1, 1, 128, 128), (16, 28, 128, 128), (3, 5, 128, 64), (257, 3, 64, 64), (7, 1, 256, 256),
    (33, 9, 80, 80), (5, 40, 512, 256), (130, 7, 128, 20), (4, 3, 128, 2), (65, 2, 20, 20),
    (2, 1, 2, 2), (9, 70, 72, 24), (1000, 17, 128, 96), (3, 2, 131, 66), (2100, 64, 128, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,rdim", SHAPES)
def test_shapes_types_and_pairings(rows, heads, dim, rdim, interleaved, dtype):
    H.say(f"[case] rotary {rows}x{heads}x{dim} R={rdim} inter={interleaved} {dtype}")
    r = Handle(dim, rdim, interleaved)
    x = randn((rows, heads, dim), dtype, 1)
    p, pd = positions_of(rows, 2)
    for backward in (False, True):
        out = torch.full_like(x, float("nan"))
        libra.libra_rotary_apply(r.h, x, pd, out, backward=backward)
        torch.cuda.synchronize()
        r.check(f64(out), f64(x), p, dtype, backward, f"backward={backward}")
    r.close()


@pytest.mark.parametrize("kw", [
    dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0, base=5e5),
    dict(scaling="bands", factor=4.0, original_length=32768, fast=32.0, slow=1.0, base=1e6,
         amplitude=1.1386294361119891),
    dict(scaling="bands", factor=8.0, original_length=8192, fast=4.0, slow=1.0)])
def test_long_contexts(kw):
    """Scaled frequencies at far positions, in float32, where an angle taken in float32 would
    be off by the position times 6e-8."""
    H.say(f"[case] rotary scaled {kw}")
    r = Handle(**kw)
    x = randn((64, 4, 128), torch.float32, 3)
    p = np.linspace(0, 2 ** 20, 64).astype(np.int32)
    out = torch.empty_like(x)
    libra.libra_rotary_apply(r.h, x, torch.from_numpy(p).cuda(), out)
    r.check(f64(out), f64(x), p, torch.float32, label=str(kw))
    r.close()


def test_positions_of_any_value():
    H.say("[case] rotary extreme positions")
    r = Handle()
    p = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -987654321, 40959], np.int32)
    x = randn((len(p), 3, 128), torch.float32, 4)
    out = torch.empty_like(x)
    libra.libra_rotary_apply(r.h, x, torch.from_numpy(p).cuda(), out)
    r.check(f64(out), f64(x), p, torch.float32)
    assert torch.equal(out[0], x[0])            # position 0 turns nothing
    r.close()


def test_given_frequencies_beyond_a_turn():
    H.say("[case] rotary given frequencies")
    f = np.array([700.25, -3.5, 0.0, 6.283185307179586, 1e6, 1e-9, 0.1, 2.0])
    r = Handle(24, 16)
    libra.libra_rotary_destroy(r.h)
    r.theta = np.asarray(f, np.longdouble)
    r.h = libra.libra_rotary_create(head_dim=24, rotary_dim=16, frequencies=f)
    x = randn((500, 3, 24), torch.float32, 5)
    p, pd = positions_of(500, 6)
    out = torch.empty_like(x)
    libra.libra_rotary_apply(r.h, x, pd, out)
    # A turn's own rounding counts here: 2^-65 turns a position, far below the slack.
    r.check(f64(out), f64(x), p, torch.float32)
    r.close()


LAYOUTS = ["packed", "heads_first", "broadcast_heads", "broadcast_rows", "odd_stride", "unaligned"]


def _view(layout, rows, heads, dim, dtype):
    """(x, out, the buffer of out) in a layout; out lies inside a buffer of fives."""
    out_buf = torch.full((rows + 3, heads + 2, dim), 5.0, dtype=dtype, device="cuda")
    out = out_buf[1:rows + 1, 1:heads + 1]
    if layout == "packed":
        x = randn((rows, heads + 6, dim), dtype, 7)[:, 3:3 + heads]
    elif layout == "heads_first":
        x = randn((heads, rows, dim), dtype, 7).transpose(0, 1)
        out_buf = torch.full((heads + 1, rows + 1, dim), 5.0, dtype=dtype, device="cuda")
        out = out_buf[:heads, :rows].transpose(0, 1)
    elif layout == "broadcast_heads":
        x = randn((rows, 1, dim), dtype, 7).expand(rows, heads, dim)
    elif layout == "broadcast_rows":
        x = randn((1, heads, dim), dtype, 7).expand(rows, heads, dim)
    elif layout == "odd_stride":
        x = randn((rows, heads, dim + 3), dtype, 7)[:, :, 1:dim + 1]
    else:
        flat = torch.full((rows * heads * dim + 1,), 5.0, dtype=dtype, device="cuda")
        x = randn((rows, heads, dim), dtype, 7)
        out_buf = flat
        out = flat[1:].view(rows, heads, dim)
    return x, out, out_buf


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rdim,interleaved", [(128, False), (64, True), (20, False)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_strides_and_untouched_surroundings(layout, rdim, interleaved, dtype):
    rows, heads, dim = 37, 6, 128
    H.say(f"[case] rotary layout {layout} R={rdim} {dtype}")
    r = Handle(dim, rdim, interleaved)
    x, out, buf = _view(layout, rows, heads, dim, dtype)
    p, pd = positions_of(rows, 8)
    libra.libra_rotary_apply(r.h, x, pd, out, backward=True)
    torch.cuda.synchronize()
    r.check(f64(out), f64(x), p, dtype, True, layout)
    out.fill_(5.0)
    assert bool((buf == 5.0).all()), "wrote outside out"
    r.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("dim,rdim,interleaved", [(128, 128, False), (128, 64, True), (80, 20, False),
                                                  (128, 22, True)])
def test_in_place_equals_out_of_place(dim, rdim, interleaved, dtype):
    H.say(f"[case] rotary in place R={rdim} {dtype}")
    r = Handle(dim, rdim, interleaved)
    buf = randn((300, 12, dim), dtype, 9)
    x = buf[:, 2:9]
    p, pd = positions_of(300, 10)
    out = torch.empty((300, 7, dim), dtype=dtype, device="cuda")
    libra.libra_rotary_apply(r.h, x, pd, out)
    rest = buf[:, [0, 1, 9, 10, 11]].clone()
    libra.libra_rotary_apply(r.h, x, pd, x)
    assert torch.equal(x, out) and torch.equal(buf[:, [0, 1, 9, 10, 11]], rest)
    r.close()


def test_gradient_against_differences():
    """y is linear in x, so a difference quotient in float64 over any step is the derivative;
    the backward pass is its transpose: <dy, y(x + v) - y(x)> = <dx, v>."""
    H.say("[case] rotary gradient")
    r = Handle(128, 96, amplitude=1.25)
    x, v, dy = (randn((50, 4, 128), torch.float32, s) for s in (11, 12, 13))
    p, pd = positions_of(50, 14)
    y0, y1, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    moved = x + v
    libra.libra_rotary_apply(r.h, x, pd, y0)
    libra.libra_rotary_apply(r.h, moved, pd, y1)
    libra.libra_rotary_apply(r.h, dy, pd, dx, backward=True)
    lhs = float((dy.double() * (y1.double() - y0.double())).sum())
    rhs = float((dx.double() * (moved.double() - x.double())).sum())
    # Each of 3 x 25,600 values is within 1.25 * 2 * 5 * (3e-7 + 6e-8) = 5e-6 of exact, and is
    # multiplied by at most 5: 3 * 25,600 * 2.5e-5 = 1.9 if all errors agreed; they are
    # independent, so sqrt(76,800) * 2.5e-5 = 7e-3.
    assert abs(lhs - rhs) < 7e-3, (lhs, rhs)
    r.check(f64(dx), f64(dy), p, torch.float32, True, "formula")
    r.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_infinities_and_nan_stay_in_their_pair(dtype):
    H.say(f"[case] rotary non-finite {dtype}")
    r = Handle(128, 64)
    x = randn((6, 2, 128), dtype, 15)
    clean = torch.empty_like(x)
    pd = torch.arange(1, 7, dtype=torch.int32, device="cuda")
    libra.libra_rotary_apply(r.h, x, pd, clean)
    bad = x.clone()
    bad[0, 0, 3], bad[1, 1, 40], bad[2, 0, 100] = float("inf"), float("nan"), float("-inf")
    out = torch.empty_like(x)
    libra.libra_rotary_apply(r.h, bad, pd, out)
    changed = (out != clean) & ~(out.isnan() & clean.isnan())
    want = torch.zeros_like(changed)
    want[0, 0, [3, 35]] = want[1, 1, [8, 40]] = want[2, 0, 100] = True
    assert torch.equal(changed, want)
    assert not out[0, 0, [3, 35]].isfinite().any() and out[1, 1, [8, 40]].isnan().all()
    assert float(out[2, 0, 100]) == float("-inf")
    r.close()


def test_offsets_past_32_bits():
    """Rows more than 2^32 bytes apart, on both sides."""
    H.say("[case] rotary far rows")
    r = Handle()
    rows, stride = 5, (1 << 29) + 64          # bf16: the last row 4.3 GB on
    x_buf = torch.empty(4 * stride + 256, dtype=torch.bfloat16, device="cuda")
    out_buf = torch.empty_like(x_buf)
    x, out = (b.as_strided((rows, 2, 128), (stride, 128, 1)) for b in (x_buf, out_buf))
    x.copy_(randn((rows, 2, 128), torch.bfloat16, 16))
    p, pd = positions_of(rows, 17)
    libra.libra_rotary_apply(r.h, x, pd, out)
    r.check(f64(out), f64(x), p, torch.bfloat16)
    r.close()


def test_rows_of_several_launches():
    """More rows than one launch takes (2^22 blocks of 256 pieces in the narrow form)."""
    H.say("[case] rotary several launches")
    dim, rdim = 512, 20
    per_launch = 2 ** 22 * 256 // (dim - rdim // 2)
    rows = per_launch + 777
    r = Handle(dim, rdim)
    x = torch.zeros((rows, 1, dim), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(x, 5.0)
    look = torch.tensor([0, 1, per_launch - 2, per_launch - 1, per_launch, per_launch + 1, rows - 1],
                        device="cuda")
    x[look] = randn((len(look), 1, dim), torch.bfloat16, 25)
    p = torch.arange(rows, dtype=torch.int32, device="cuda") % 5000
    libra.libra_rotary_apply(r.h, x, p, out)
    torch.cuda.synchronize()
    r.check(f64(out[look]), f64(x[look]), p[look].cpu().numpy(), torch.bfloat16)
    assert not bool((out == 5.0).any())
    r.close()


def test_other_stream_and_graph_with_new_positions():
    H.say("[case] rotary stream and graph")
    r = Handle(128, 128, True)
    x = randn((100, 8, 128), torch.bfloat16, 18)
    out = torch.empty_like(x)
    p, pd = positions_of(100, 19)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    libra.libra_rotary_apply(r.h, x, pd, out, stream=side)
    side.synchronize()
    r.check(f64(out), f64(x), p, torch.bfloat16)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        libra.libra_rotary_apply(r.h, x, pd, out)
    for seed in (20, 21, 22):
        p, new = positions_of(100, seed)
        pd.copy_(new)
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        r.check(f64(out), f64(x), p, torch.bfloat16, label="replay")
        eager = torch.empty_like(out)
        libra.libra_rotary_apply(r.h, x, pd, eager)
        assert torch.equal(eager, out)
    r.close()


def test_refusals_of_the_binding():
    r = Handle()
    x = randn((4, 2, 128), torch.bfloat16, 23)
    _, pd = positions_of(4, 24)
    for bad in (lambda: libra.libra_rotary_apply(r.h, x, pd[:3], x),
                lambda: libra.libra_rotary_apply(r.h, x, pd.long(), x),
                lambda: libra.libra_rotary_apply(r.h, x, pd, x.float()),
                lambda: libra.libra_rotary_apply(r.h, x, pd.cpu(), x),
                lambda: libra.libra_rotary_apply(r.h, x[:, :, :64], pd, x[:, :, :64]),
                lambda: libra.libra_rotary_apply(r.h, x.double(), pd, x.double()),
                lambda: libra.libra_rotary_apply(r.h, x, pd, x.cpu())):
        with pytest.raises((ValueError, libra.LibraError)):
            bad()
    r.close()
