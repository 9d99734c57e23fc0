"""No launch is larger than a HIP grid holds (CPU: the HIP calls of the library are taken by
the driver `tests/sanitize/launch_sizes_main.cpp`, nothing is launched): the entry points at
the largest sizes that they accept."""
import os
import shutil
import subprocess

import pytest

from paper_2607_08782_amd import moe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("group", ["mxfp4", "packaging", "gradients"])
def test_every_launch_fits_a_grid(tmp_path, group):
    if not os.path.exists(moe.LIB_PATH):
        from paper_2607_08782_amd import build
        build.build()
    exe = str(tmp_path / "launch_sizes")
    # -rdynamic: the driver's definitions come before the runtime's
    subprocess.run(["g++", "-O1", "-std=c++17", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "sanitize", "launch_sizes_main.cpp"), "-o", exe, "-ldl"],
                   check=True, timeout=120)
    r = subprocess.run([exe, moe.LIB_PATH, group], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "launch sizes: OK" in r.stdout, r.stdout + r.stderr[-3000:]
