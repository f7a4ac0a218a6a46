"""The largest calls of the paged cache, with the library's host code run on the CPU over a stand-in for the HIP runtime: no launch
may be larger than a grid can be."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB_DIR = os.path.join(ROOT, "paper_2603_04716_amd")


def test_calls_at_the_size_limits(tmp_path):
    exe = str(tmp_path / "driver")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wno-missing-field-initializers", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include",
                    "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "paged_launches_driver.cpp"),
                    os.path.join(LIB_DIR, "libpd_mi355x.so"), "-rdynamic", f"-Wl,-rpath,{LIB_DIR}",
                    "-Wl,--unresolved-symbols=ignore-in-shared-libs", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
