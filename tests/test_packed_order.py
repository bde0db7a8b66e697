"""Host check of the packed backward's order (csrc/packed_order.h), against
enumeration: a chain's blocks, a block's last tile, and that chains start longest first
with each sequence's own in ascending order (what keeps their waits from a cycle)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_packed_order(tmp_path):
    exe = tmp_path / "packed_order_check"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2601_21824_amd", "csrc"),
                    os.path.join(ROOT, "tests", "packed_order_check.cpp"), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    print(res.stdout)
    assert res.returncode == 0, res.stdout
