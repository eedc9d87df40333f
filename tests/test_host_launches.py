"""The library's launches at its largest sizes, noted by a program that stands in for the HIP runtime.  Nothing runs on a GPU."""
import os
import subprocess

from paper_2402_14800_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_launches_keep_to_the_grid_limits(tmp_path):
    exe, lib = str(tmp_path / "host_launch_driver"), binding.library_path()
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "host_launch_driver.cpp"), "-o", exe, lib, "-Wl,-rpath," + os.path.dirname(lib),
                        "-Wl,-rpath-link,/opt/rocm/lib", "-Wl,-rpath,/opt/rocm/lib", "-Wl,--unresolved-symbols=ignore-in-shared-libs"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "all checks passed", (r.stdout[-4000:], r.stderr[-2000:])
