"""The merge of recomputed attention weights takes the CTAs whose parts it adds from device memory; a CTA that gave up
a wait leaves some of it unwritten, and then no part past the last CTA's may be read (tests/cuda/split_check.cu, built
with nvcc; its checks run on the host)."""
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2609_04971_gb300", "csrc")


def test_parts_of_split_items_stay_in_range(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    exe = str(tmp_path / "split_check")
    subprocess.check_call([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-O2", "-std=c++17", "-I", CSRC, "-I",
                           os.path.join(ROOT, "include"), "-o", exe, os.path.join(HERE, "cuda", "split_check.cu")])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    print(out.stdout)
    assert out.returncode == 0, out.stdout + out.stderr
