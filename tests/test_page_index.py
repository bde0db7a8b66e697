"""Host check of the paged cache's index arithmetic (csrc/page_index.h), which the
append and the one-token attention kernels use as it is: tables that hold pages
outside the cache, places outside the table, and the split into chunks."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_page_index(tmp_path):
    exe = tmp_path / "page_index_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2601_21824_amd", "csrc"),
                    os.path.join(ROOT, "tests", "page_index_check.cpp"), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    print(res.stdout)
    assert res.returncode == 0, res.stdout
