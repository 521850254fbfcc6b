"""A warp of the attention over 4-bit caches waits for its tiles of a ring that it shares with others, by the parity of a
phase: no order in which copies land may let it read another tile or stop it (tests/cuda/ring_check.cpp, a model of the
ring on the host with the walk of the kernel, k_ring4.cuh)."""
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_04971_gb300", "csrc")


def test_no_tile_is_read_early_and_no_warp_stops(tmp_path):
    exe = str(tmp_path / "ring_check")
    subprocess.check_call([shutil.which("g++") or "g++", "-O2", "-std=c++17", "-I", CSRC, "-o", exe,
                           os.path.join(HERE, "cuda", "ring_check.cpp")])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    print(out.stdout)
    assert out.returncode == 0, out.stdout + out.stderr


def test_the_kernel_walks_by_it():
    src = open(os.path.join(CSRC, "k_attend4.cu")).read()
    assert "RingWalk<typename C::Ring>" in src
    for call in ("ring_at.there(", "ring_at.await(", "try_wait(&full_bar[", "at_wait(&full_bar["):
        assert src.count(call) == 1, call  # a step's tile is waited for nowhere else
