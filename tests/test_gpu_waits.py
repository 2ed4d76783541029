"""Waits inside a kernel that run out: the kernels end, say so, and leave the GPU as usable as it was. A library is compiled whose waits have no tries, or
one or a few, so that they run out while every copy and product that they wait for completes as ever."""
import os
import subprocess
import sys

import pytest

from paper_2410_05076_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2410_05076_b200 import binding, build
build.LIB, build.is_stale = {lib!r}, lambda: False
from tests.test_gpu_blocks import make
from tests.test_gpu_prompt import chunk_inputs
td = binding.Tidal(0)
seen = set()
for layout, fp8 in (("paged", False), ("hnd", True)):
    for lens, new, hq, hkv in (([5000], [7], 8, 2), ([700, 300, 1], [300, 1, 1], 8, 2), ([4000] * 40, [200] * 40, 6, 2), ([900], [900], 16, 16)):
        lay = make(lens, hq, hkv, layout, fp8, seed=1)
        q, off = chunk_inputs(lay, new)
        lse = torch.zeros(sum(new), hq, device="cuda")
        w = torch.zeros(len(lens), hkv, lay.max_ctx_len, device="cuda")
        one = torch.zeros(len(lens), 1, lay.max_ctx_len, device="cuda")
        for call in (lambda: td.chunk_attn(lay, q, off, lse=lse), lambda: td.chunk_attn(lay, q, off, lse=lse, window=100),
                     lambda: td.chunk_weights(lay, q, off, lse, w), lambda: td.chunk_weights(lay, q, off, lse, one)):
            call()
            seen.add(td.device_status())
            assert td.device_status() == binding.OK
print("seen", sorted(seen))
"""


@pytest.fixture(scope="module")
def libraries(tmp_path_factory):
    at = tmp_path_factory.mktemp("waits")
    jobs = {}
    for tries in (0, 1, 4):
        path = str(at / f"waits{tries}.so")
        jobs[tries] = path, subprocess.Popen([build.nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-cudart", "static",
                                              f"-DTIDAL_WAIT_TRIES={tries}", "-o", path, os.path.join(build.CSRC, "tidal_api.cu")], stderr=subprocess.DEVNULL)
    assert all(p.wait(600) == 0 for _, p in jobs.values())
    return {tries: path for tries, (path, _) in jobs.items()}


@pytest.mark.parametrize("tries", [0, 1, 4])
def test_kernels_whose_waits_run_out_end_and_say_so(libraries, tries):
    r = subprocess.run([sys.executable, "-c", CODE.format(root=ROOT, lib=libraries[tries])], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    seen = r.stdout.strip().splitlines()[-1]
    assert "-5" in seen if tries == 0 else seen in ("seen [-5]", "seen [-5, 0]", "seen [0]"), seen
