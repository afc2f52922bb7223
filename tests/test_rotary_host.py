"""Host side of the rotary operators (no GPU): handles, their frequencies, and every refusal,
which comes before any HIP call."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import rotary as ref
from paper_2606_03077_amd import libra

INVAL, UNSUPPORTED, WORKSPACE = 1, 2, 3
SCALINGS = {"plain": libra.LIBRA_ROTARY_PLAIN, "linear": libra.LIBRA_ROTARY_LINEAR,
            "base": libra.LIBRA_ROTARY_BASE, "bands": libra.LIBRA_ROTARY_BANDS}
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def refused(status, fn, *args, **kw):
    with pytest.raises(libra.LibraError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)


@pytest.mark.parametrize("rdim", [2, 20, 64, 128, 256])
@pytest.mark.parametrize("kw", [
    dict(), dict(base=1e6), dict(scaling="linear", factor=8.0),
    dict(scaling="base", factor=4.0), dict(scaling="bands", factor=4.0, original_length=32768,
                                           fast=32.0, slow=1.0),
    dict(scaling="bands", factor=8.0, original_length=8192, fast=4.0, slow=1.0, base=5e5)])
def test_frequencies(rdim, kw):
    if rdim == 2 and kw.get("scaling") == "base":
        kw = dict(kw, scaling="linear")
    h = libra.libra_rotary_create(head_dim=256, rotary_dim=rdim, amplitude=1.25,
                                  **dict(kw, scaling=SCALINGS[kw.get("scaling", "plain")]))
    got = libra.libra_rotary_get(h)
    libra.libra_rotary_destroy(h)
    want = ref.frequencies(rdim, **kw).astype(np.float64)
    assert got["rotary_dim"] == rdim and got["amplitude"] == 1.25
    # Both are taken in long double and rounded once: equal but for that rounding's edge.
    np.testing.assert_allclose(got["frequencies"], want, rtol=2 * np.finfo(np.float64).eps)


def test_given_frequencies():
    f = np.array([1.0, -0.5, 0.0, 700.25])
    h = libra.libra_rotary_create(head_dim=10, rotary_dim=8, frequencies=f, base=0.0)
    assert np.array_equal(libra.libra_rotary_get(h)["frequencies"], f)
    libra.libra_rotary_destroy(h)
    h = libra.libra_rotary_create(rotary_dim=8, frequencies=f, scaling=SCALINGS["linear"], factor=2.0)
    assert np.array_equal(libra.libra_rotary_get(h)["frequencies"], f / 2)
    libra.libra_rotary_destroy(h)
    with pytest.raises(ValueError):
        libra.libra_rotary_create(rotary_dim=8, frequencies=f[:3])


def test_default_is_the_whole_head():
    h = libra.libra_rotary_create()
    assert libra.libra_rotary_get(h)["rotary_dim"] == 128
    assert libra.libra_rotary_get(h)["amplitude"] == 1.0
    libra.libra_rotary_destroy(h)


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=0), UNSUPPORTED), (dict(head_dim=514), UNSUPPORTED),
    (dict(rotary_dim=3), INVAL), (dict(rotary_dim=130), INVAL), (dict(rotary_dim=-2), INVAL),
    (dict(head_dim=300, rotary_dim=258), UNSUPPORTED), (dict(head_dim=127), INVAL),
    (dict(pairing=2), INVAL), (dict(pairing=-1), INVAL), (dict(scaling=4), INVAL),
    (dict(base=0.0), INVAL), (dict(base=-1.0), INVAL), (dict(base=float("nan")), INVAL),
    (dict(base=float("inf")), INVAL), (dict(base=1e-40), INVAL),
    (dict(scaling=1, factor=0.0), INVAL), (dict(scaling=1, factor=float("nan")), INVAL),
    (dict(scaling=2, factor=-2.0), INVAL), (dict(scaling=2, factor=2.0, rotary_dim=2), INVAL),
    (dict(scaling=2, factor=2.0, rotary_dim=4, frequencies=[1.0, 0.5]), INVAL),
    (dict(scaling=3, factor=2.0, fast=2.0), INVAL),
    (dict(scaling=3, factor=2.0, original_length=100, fast=1.0, slow=1.0), INVAL),
    (dict(scaling=3, factor=2.0, original_length=100, fast=2.0, slow=-1.0), INVAL),
    (dict(scaling=3, factor=2.0, original_length=100, fast=float("inf")), INVAL),
    (dict(amplitude=-1.0), INVAL), (dict(amplitude=float("nan")), INVAL),
    (dict(amplitude=1e300), INVAL), (dict(amplitude=1e-300), INVAL),
    (dict(rotary_dim=4, frequencies=[1.0, float("nan")]), INVAL),
    (dict(rotary_dim=4, frequencies=[1.0, float("inf")]), INVAL),
    (dict(rotary_dim=4, frequencies=[1.0, 2e6]), INVAL)])
def test_refused_handles(kw, status):
    refused(status, libra.libra_rotary_create, **kw)


def _raw(name, *args):
    lib = libra.load()
    fn = getattr(lib, name)
    return fn(*[a if not isinstance(a, float) else ctypes.c_float(a) for a in args])


P = 0x10000   # never read: the host refuses first


@pytest.fixture()
def rotary():
    h = libra.libra_rotary_create()
    yield h
    libra.libra_rotary_destroy(h)


def _apply(h, dtype=0, x=P, xr=256, xh=128, pos=P, rows=3, heads=2, dim=128, out=2 * P, outr=256,
           outh=128):
    return _raw("libra_rotary_apply", h, dtype, x, xr, xh, pos, rows, heads, dim, 0, out, outr, outh,
                None)


@pytest.mark.parametrize("kw,status", [
    (dict(dim=64), INVAL), (dict(dim=256), INVAL), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(rows=-1), INVAL),
    (dict(heads=-1), INVAL), (dict(rows=2 ** 31), UNSUPPORTED), (dict(heads=65536), UNSUPPORTED),
    (dict(x=None), INVAL), (dict(out=None), INVAL), (dict(pos=None), INVAL),
    (dict(x=P + 1), INVAL), (dict(dtype=2, out=P + 2), INVAL), (dict(xr=-128), INVAL),
    (dict(xh=-1), INVAL), (dict(outr=-256), INVAL), (dict(outh=127), INVAL), (dict(outr=255), INVAL),
    (dict(outr=0), INVAL), (dict(outh=0), INVAL), (dict(xr=2 ** 56), INVAL),
    (dict(rows=2 ** 31 - 1, outr=2 ** 40), INVAL), (dict(out=P, outr=384), INVAL),
    (dict(out=P, outh=129, outr=512), INVAL)])
def test_refused_apply(rotary, kw, status):
    assert _apply(rotary, **kw) == status


def test_apply_without_rows_is_no_call(rotary):
    assert _apply(rotary, rows=0, x=None, out=None, pos=None) == 0
    assert _apply(rotary, heads=0, x=None, out=None, pos=None) == 0
    assert _apply(None) == INVAL


def _layout(hkv=2):
    return libra.libra_kv_layout_create(P, P, 10, hkv)


def _append(layout, h, pos=P, slots=P, rows=3, q=None, qr=0, hq=0, k=P, kr=256, v=P, vr=256, hkv=2, q_out=None):
    return _raw("libra_kv_append", layout, h, pos, slots, rows, q, qr, hq, k, kr, v, vr, hkv, q_out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVAL), (dict(rows=2 ** 31), UNSUPPORTED), (dict(slots=None), INVAL),
    (dict(hkv=1), INVAL), (dict(hkv=4, kr=512, vr=512), INVAL),
    (dict(pos=None), INVAL), (dict(k=None), INVAL), (dict(v=None), INVAL), (dict(k=P + 8), INVAL),
    (dict(v=P + 2), INVAL), (dict(kr=255), INVAL), (dict(kr=248), INVAL), (dict(vr=0), INVAL),
    (dict(vr=-256), INVAL), (dict(vr=2 ** 60), INVAL), (dict(q=P, qr=512, hq=4), INVAL),
    (dict(q_out=P, qr=512, hq=4), INVAL), (dict(q=P, qr=512, hq=0, q_out=P), INVAL),
    (dict(q=P, qr=504, hq=4, q_out=P), INVAL), (dict(q=P, qr=512, hq=4, q_out=P + 8), INVAL),
    (dict(q=P, qr=640, hq=4, q_out=P), INVAL), (dict(q=P, qr=512, hq=65536, q_out=P), INVAL)])
def test_refused_kv_append(rotary, kw, status):
    lay = _layout()
    assert _append(lay, rotary, **kw) == status
    libra.libra_kv_layout_destroy(lay)


def test_kv_append_other_refusals(rotary):
    lay = _layout()
    assert _append(None, rotary) == INVAL
    assert _append(lay, None, q=P, qr=512, hq=4, q_out=P) == INVAL   # q needs a rotary
    assert _append(lay, rotary, rows=0, slots=None, pos=None, k=None, v=None) == 0
    other = libra.libra_rotary_create(head_dim=64)
    assert _append(lay, other) == INVAL                              # not the cache's heads
    libra.libra_rotary_destroy(other)
    libra.libra_kv_layout_destroy(lay)


def test_refused_append_attn(rotary):
    lay = _layout()
    plan = libra.libra_splitkv_plan(libra.LIBRA_MODE_APPEND, 2, 4, 2, [20, 5], [3, 1], num_cus=8)
    decode = libra.libra_splitkv_plan(libra.LIBRA_MODE_DECODE, 2, 4, 2, [20, 5], None, num_cus=8)
    other = libra.libra_rotary_create(head_dim=64)

    def call(plan=plan, h=rotary, pos=None, rows=4, q=P, qr=512, k=P, kr=256, v=P, vr=256, bt=P, stride=2,
             batch=2, hq=4, hkv=2, scale=0.1, ws=P, n=1 << 30, out=P):
        return _raw("libra_append_attn_rotary", lay, plan, h, pos, rows, q, qr, k, kr, v, vr, hkv, bt,
                    stride, batch, hq, scale, 0, ws, n, out, None, None)

    for kw, status in [(dict(plan=decode), INVAL), (dict(plan=None), INVAL), (dict(h=None), INVAL),
                       (dict(h=other), INVAL), (dict(rows=3), INVAL), (dict(rows=0), INVAL),
                       (dict(q=None), INVAL), (dict(q=P + 8), INVAL),
                       (dict(qr=511), INVAL), (dict(qr=256), INVAL), (dict(k=None), INVAL),
                       (dict(kr=128), INVAL), (dict(v=P + 4), INVAL), (dict(vr=300), INVAL),
                       (dict(bt=None), INVAL), (dict(stride=1), INVAL), (dict(batch=1), INVAL),
                       (dict(hq=8), INVAL), (dict(hkv=1), INVAL), (dict(hkv=4, kr=512, vr=512), INVAL), (dict(scale=0.0), INVAL), (dict(scale=float("nan")), INVAL),
                       (dict(ws=None), INVAL), (dict(ws=P + 16), INVAL), (dict(n=16), WORKSPACE),
                       (dict(out=P + 2), INVAL), (dict(out=None), INVAL)]:
        assert call(**kw) == status, (kw, libra.libra_last_error())
    libra.libra_rotary_destroy(other)
    libra.libra_plan_destroy(decode)
    libra.libra_plan_destroy(plan)
    libra.libra_kv_layout_destroy(lay)


def test_tensors_of_another_device_are_refused(rotary, monkeypatch):
    """The binding refuses what does not lie on the current device, before the library is called."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(libra, "_stream", lambda *a: None)
    x, pos = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    lay = _layout()
    for bad in (lambda: libra.libra_rotary_apply(rotary, x, pos, x),
                lambda: libra.libra_kv_append(lay, rotary, pos, pos.long(), None, x, x, None),
                lambda: libra.libra_append_attn_rotary(lay, None, rotary, pos, x, x, x, pos, 1, 1, 2,
                                                       0.1, pos, x)):
        with pytest.raises(ValueError, match="current device"):
            bad()
    libra.libra_kv_layout_destroy(lay)


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the ROCm headers")
def test_host_calls_are_clean_and_allocate_nothing(tmp_path):
    """The rotary entry points against the counting HIP stand-in, under the sanitizers."""
    exe = str(tmp_path / "rotary_host")
    asan = os.path.join(ROOT, "tests", "host_asan")
    csrc = os.path.join(ROOT, "paper_2606_03077_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__",
           "-DLIBRA_STUB_LAUNCH_OK", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
           "-I" + csrc, "-I" + asan]
    cmd += [os.path.join(csrc, f) for f in ("api.cpp", "plan.cpp", "migrate.cpp", "cost_model.cpp",
                                            "scheduler.cpp", "positions.cpp")]
    cmd += [os.path.join(asan, f) for f in ("stubs.cpp", "fake_hip.cpp", "rotary_driver.cpp")]
    cmd += ["-pthread", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"), timeout=300)
    assert r.returncode == 0 and "rotary host ok" in r.stdout, (r.stdout + r.stderr)[-4000:]
