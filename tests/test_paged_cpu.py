"""The kernels of the paged cache compiled for the CPU (tests/cpu_hip,
tests/paged_cpu.cpp): batches whose pages, rows or lengths are out of range stay
inside their buffers, and the rest of them is right."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"


@pytest.mark.skipif(not os.path.exists(CLANG), reason="needs clang++")
def test_batches_out_of_range_stay_in_bounds(tmp_path):
    exe = str(tmp_path / "paged_cpu")
    r = subprocess.run([CLANG, "-std=c++17", "-O1", "-I", os.path.join(HERE, "cpu_hip"),
                        os.path.join(HERE, "paged_cpu.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stdout[-500:])


@pytest.mark.skipif(not os.path.exists(CLANG), reason="needs clang++")
def test_values_at_which_the_way_to_a_result_shows(tmp_path):
    exe = str(tmp_path / "paged_values_cpu")
    r = subprocess.run([CLANG, "-std=c++17", "-O2", "-w", "-I", os.path.join(HERE, "cpu_hip"),
                        os.path.join(HERE, "paged_values_cpu.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.returncode, r.stdout[-500:])
