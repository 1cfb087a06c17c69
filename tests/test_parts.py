"""Host checks of csrc/sfmp_parts.h, which the attention kernels include: equal parts of up to 2^31 - 1 pages."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def test_parts_of_any_number_of_pages(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "parts_driver")
    r = subprocess.run([gxx, "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan",
                        os.path.join(HERE, "parts_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr
