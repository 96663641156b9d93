"""The operators' C entry points let no C++ exception out where host memory is short: tests/operators_memory_check.cpp, whose allocations fail one
after the other, built with g++ against the in-tree library."""
import os
import subprocess

from paper_2410_11415_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_exception_comes_out(tmp_path):
    exe, lib = str(tmp_path / "operators_memory_check"), binding.library_path()
    binding.load()
    subprocess.run(["g++", "-std=c++17", "-Wall", "-o", exe, os.path.join(ROOT, "tests", "operators_memory_check.cpp"), lib, "-L/opt/rocm/lib",
                    "-lamdhip64", "-Wl,-rpath," + os.path.dirname(lib), "-Wl,-rpath,/opt/rocm/lib"], check=True, cwd=ROOT)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr
