"""Angles of large frequencies and far positions, against integer arithmetic.

A given frequency is a float64, so its turns theta / 2 pi mod 1 are an exact fraction of pi's
digits; the handle holds them in units of 2^-64, rounded to nearest, whatever the frequency."""
import os
import random
import shutil
import subprocess
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2606_03077_amd import libra

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899,
              10 ** 80)
FREQUENCIES = [1e6, -1e6, 999999.1, 12345.678, -700.25, 6.283185307179586, 3.0, 1.0, 0.1,
               2.0 ** -30, 5e-324, 0.0, 1e-9, -1e-9]


def turns(theta):
    """theta / 2 pi as a fraction, good to 60 digits."""
    return Fraction(theta) / (2 * PI)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_turns_of_any_frequency(tmp_path):
    exe = str(tmp_path / "turns")
    cmd = ["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I" + os.path.join(ROOT, "paper_2606_03077_amd", "csrc"),
           os.path.join(ROOT, "tests", "host_asan", "turns_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    rng = random.Random(9)
    theta = FREQUENCIES + [rng.choice([-1, 1]) * 10.0 ** rng.uniform(-25, 6) for _ in range(5000)]
    r = subprocess.run([exe], input="\n".join(t.hex() for t in theta) + "\n", capture_output=True,
                       text=True, timeout=60)
    assert r.returncode == 0, r.stderr[-4000:]
    got = [int(line) for line in r.stdout.split()]
    assert len(got) == len(theta)
    for t, g in zip(theta, got):
        off = (turns(t) * 2 ** 64 - g) % 2 ** 64
        # Half a unit, and what the constant's 192 bits leave out.
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 2 ** 40), t


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_far_positions_of_large_frequencies(dtype):
    """|y - exact| <= 3e-7 of the pair's size (test_gpu_rotary.py derives it) and the angle's
    2^31 * 2^-65 turns, 4e-10 radians, then half a step of the type."""
    f = np.array([t for t in FREQUENCIES if t])
    p = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -987654321, 40960, 0], np.int32)
    half = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}[dtype]
    n = len(f)
    h = libra.libra_rotary_create(head_dim=2 * n, rotary_dim=2 * n, frequencies=f)
    g = torch.Generator(device="cuda").manual_seed(31)
    x = torch.randn((len(p), 2, 2 * n), dtype=dtype, device="cuda", generator=g)
    out = torch.empty_like(x)
    libra.libra_rotary_apply(h, x, torch.from_numpy(p).cuda(), out)
    a, y = x.double().cpu().numpy(), out.double().cpu().numpy()
    libra.libra_rotary_destroy(h)
    angle = np.array([[float(turns(t) * int(q) % 1) for t in f] for q in p]) * (2 * np.pi)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    x1, x2 = a[..., :n], a[..., n:]
    want = np.concatenate([x1 * c - x2 * s, x2 * c + x1 * s], axis=-1)
    size = np.tile(np.abs(x1) + np.abs(x2), 2)
    slack = (3e-7 + 4e-10) * size
    assert (np.abs(y - want) <= slack + half * (np.abs(want) + slack)).all()
