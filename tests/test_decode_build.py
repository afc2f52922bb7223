"""The decode kernels' workgroup is four waves, which their turned rows in LDS need, whatever the
compiler is told."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which("hipcc") is None, reason="needs hipcc")
def test_waves_of_the_decode_kernels(tmp_path):
    src = tmp_path / "waves.hip"
    src.write_text('#include "decode.hip"\n'
                   'static_assert(libra::kWaves == 4 && libra::kThreads == 256, "four waves");\n')
    r = subprocess.run([HIPCC if os.path.exists(HIPCC) else "hipcc", "-std=c++17", "-fsyntax-only",
                        "--cuda-host-only", "--offload-arch=gfx950", "-DLIBRA_DECODE_WAVES=8",
                        "-I" + os.path.join(ROOT, "include"),
                        "-I" + os.path.join(ROOT, "paper_2606_03077_amd", "csrc"), str(src)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
