"""The microscaled formats' scale, by a host program over every bf16 value, and the tests' own reference of the elements."""
import os
import subprocess

import torch

import mx_util

HERE = os.path.dirname(os.path.abspath(__file__))


def test_scale_bytes(tmp_path):
    exe = str(tmp_path / "mx_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(HERE, "..", "paper_2601_21824_amd", "csrc"),
                    os.path.join(HERE, "mx_check.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout


def test_reference_is_the_nearest_element():
    g = torch.Generator()
    g.manual_seed(1)
    x = torch.randn(500, 64, generator=g) * 2.0 ** torch.randint(-30, 30, (500, 1), generator=g)
    for kind in ("mxfp8", "mxfp4"):
        code, byte, odd = mx_util.quantise64(x, kind)
        s = torch.exp2(byte.double() - 127).repeat_interleave(32, -1)
        y, grid = x.double() / s, mx_util.grid(kind)
        got = mx_util.values64(mx_util.pack(code, kind), byte, kind) / s
        assert not odd.any() and bool((y.abs() <= grid[-1]).all())
        assert torch.equal((got - y).abs(), (y.abs()[..., None] - grid).abs().amin(-1))
        half = byte.int() - 1  # the scale's half does not hold the block
        assert bool((x.double().unflatten(-1, (-1, 32)).abs().amax(-1) > grid[-1] * torch.exp2(half.double() - 127)).all())
    assert torch.equal(code.new_tensor([2, 0]), mx_util.quantise64(torch.tensor([0.75, 0.25] + [6.0] + [0.0] * 29), "mxfp4")[0][:2])
