"""The division of a paged attention call of many rows over its workgroups, on the CPU: the kernel's own arithmetic
(csrc/paged_division.h) has to give every tile of keys to one workgroup, in small calls and in the largest that the entry point takes."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("division") / "driver")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                    "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "paper_2603_04716_amd", "csrc"),
                    os.path.join(ROOT, "tests", "paged_division_driver.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("case", ["quotients", "small", "large"])
def test_division(driver, case):
    r = subprocess.run([driver, case], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
