"""The waits of the latent kernel's load warps, followed through every order of events on the CPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_load_warp_passes_a_release_early(tmp_path):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    if not os.path.exists(nvcc) and shutil.which("nvcc") is None:
        pytest.skip("nvcc not available")
    exe = str(tmp_path / "latent_ring_check")
    subprocess.check_call([nvcc, "-O2", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a",
                           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2607_28633_b200", "csrc"),
                           os.path.join(ROOT, "tests", "native", "latent_ring_check.cu"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr


def test_dependents_are_released_behind_the_allocation():
    """A CTA of the launch behind may hold tensor memory while it waits for this grid to end. It must
    not start before every CTA of this grid has its own: a warp of one that is still asking for it would
    wait for the other for good."""
    with open(os.path.join(ROOT, "paper_2607_28633_b200", "csrc", "topkv_latent.cuh")) as f:
        kernel = f.read().split("topkv_latent_kernel(const AttendParams p", 1)[1]
    asked = kernel.index("tcgen05.alloc")
    granted = kernel.index("__syncthreads();", asked)   # the allocating warp arrives with its memory
    assert kernel.count("pdl_release_next_grid();") == 1 and kernel.index("pdl_release_next_grid();") > granted
