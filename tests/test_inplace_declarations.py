"""moe_permute_backward may write dx over dx_add (CPU): its kernels must not be told that the
two do not overlap.  The sources are compiled to the compiler's own form for gfx950, unoptimised,
and the kernels' declarations read."""
import os
import re
import subprocess

import pytest

from paper_2607_08782_amd import build


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
def test_kernels_of_the_packaging_gradient_may_work_in_place(tmp_path):
    out = str(tmp_path / "device.ll")
    flags = [f for f in build.CFLAGS if f != "-O3"] + ["-O1", "-Xclang", "-disable-llvm-passes"]
    r = subprocess.run([build.HIPCC] + flags + ["--offload-device-only", "-emit-llvm", "-S",
                                                os.path.join(build.CSRC, "combine.hip"), "-o", out],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    kernels = re.findall(r"^define .*amdgpu_kernel void @\S*combine\w*?kernel\w*\((.*?)\) #", open(out).read(), re.M)
    assert len(kernels) >= 12
    for params in kernels:
        params = params.split(", ")
        pointers = [p for p in params if p.startswith("ptr")]
        # y_perm, token_row, gate, y_shared (dx_add) and y (dx), in order
        assert len(pointers) == 5 and params[-1] == pointers[-1]
        assert ["noalias" in p for p in pointers] == [True, True, True, False, False], params
