"""The arithmetic of the pages (csrc/pages.h) on the host, under the sanitizers: exponents, places, and who works on what in a decode step."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_page_arithmetic(tmp_path):
    exe = str(tmp_path / "pages")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
                    "-static-libasan", "-I", os.path.join(os.path.dirname(HERE), "paper_2604_16734_amd", "csrc"),
                    os.path.join(HERE, "host_asan", "pages.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr
