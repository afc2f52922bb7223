"""Strides of libra_rotary_apply's output: whatever overlaps itself is refused (on the host, before
any HIP call), whatever does not is taken."""
import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra

import gpu_harness as H
from test_gpu_rotary import Handle, f64, randn

N = 8                       # channels of a head on the host's side


def starts(rows, heads, row, head):
    return np.sort((np.arange(rows)[:, None] * row + np.arange(heads)[None] * head).ravel())


def test_every_small_layout():
    """The call is refused in any case, so that none reaches a launch: for its strides, or else as
    in place with the strides of x (4 elements, which no output can have) differing."""
    h, lib, taken = libra.libra_rotary_create(head_dim=N), libra.load(), 0
    for rows, heads in [(1, 3), (2, 1), (2, 2), (2, 4), (3, 2), (3, 4), (5, 3), (5, 4)]:
        for row in range(44):
            for head in range(44):
                status = lib.libra_rotary_apply(h, libra.LIBRA_DTYPE_FP32, 0x10000, 4, 4, 0x10000, rows,
                                                heads, N, 0, 0x10000, row, head, None)
                assert status == 1
                want = "overlap" if (np.diff(starts(rows, heads, row, head)) < N).any() else "in place"
                assert want in libra.libra_last_error(), (rows, heads, row, head)
                taken += want == "in place"
    assert taken > 1000
    libra.libra_rotary_destroy(h)


def test_many_heads_between_few_rows():
    """65,535 heads, and a second row near the first heads or the last ones."""
    h, lib = libra.libra_rotary_create(head_dim=N), libra.load()
    for row, head, want in [(12, 16, "overlap"), (12, 24, "in place"), (3 * 65534 * 8 + 4, 24, "overlap"),
                            (3 * 65534 * 8 + 8, 24, "in place"), (3 * 65533 * 8 + 16, 24, "in place")]:
        status = lib.libra_rotary_apply(h, libra.LIBRA_DTYPE_FP32, 0x10000, 4, 4, 0x10000, 2, 65535, N, 0,
                                        0x10000, row, head, None)
        assert status == 1 and want in libra.libra_last_error(), (row, head)
    libra.libra_rotary_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,heads,row,head", [(2, 2, 384, 256), (3, 5, 128, 384), (4, 3, 256, 1152),
                                                 (2, 7, 130, 260)])
@pytest.mark.parametrize("rdim", [128, 20])
def test_woven_rows(rows, heads, row, head, rdim):
    """Rows whose heads lie between those of other rows."""
    H.say(f"[case] rotary woven {rows}x{heads} at {row}, {head}, R={rdim}")
    at = starts(rows, heads, row, head)
    assert (np.diff(at) >= 128).all()
    r = Handle(rdim=rdim)
    x = randn((rows, heads, 128), torch.bfloat16, 41)
    buf = torch.full((int(at[-1]) + 200,), 5.0, dtype=torch.bfloat16, device="cuda")
    out = buf.as_strided((rows, heads, 128), (row, head, 1))
    p = np.arange(rows, dtype=np.int32) + 100
    libra.libra_rotary_apply(r.h, x, torch.from_numpy(p).cuda(), out)
    r.check(f64(out), f64(x), p, torch.bfloat16, label="woven")
    first = out.clone()
    out.copy_(x)
    libra.libra_rotary_apply(r.h, out, torch.from_numpy(p).cuda(), out)
    assert torch.equal(out, first)
    out.fill_(5.0)
    assert bool((buf == 5.0).all())
    r.close()
