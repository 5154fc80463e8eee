"""What the compiler makes of the kernels of the losses and of many tensors: their gfx950 assembly, read on the CPU."""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2512_17570_amd import build as B


@pytest.fixture(scope="module", params=["gs_loss.hip", "gs_tensors.hip"])
def kernels(request, tmp_path_factory):
    """{name with template arguments: (registers of a lane, bytes of arguments, lanes of its workgroups, assembly)}"""
    out = str(tmp_path_factory.mktemp("asm") / "kernels.s")
    flags = [f for f in B.FLAGS if f != "-shared"]
    subprocess.run([B.HIPCC, *flags, "--offload-device-only", "-S", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC,
                    os.path.join(B.CSRC, request.param), "-o", out], check=True, capture_output=True, text=True)
    text = open(out).read()
    found = {}
    for name, block in re.findall(r"\.amdhsa_kernel (\S+)\n(.*?)\.end_amdhsa_kernel", text, re.S):
        number = lambda key: int(re.search(rf"{key} (\d+)", block)[1])  # noqa: E731
        start = text.index(f"\n{name}:")
        code = text[start:text.index(".section", start)]
        lanes = int(re.search(rf"\.max_flat_workgroup_size: (\d+)\n(?:.*\n)*?.*\.name: +{re.escape(name)}\n", text)[1])
        found[name] = number("next_free_vgpr"), number("kernarg_size"), number("private_segment_fixed_size"), lanes, code
    assert found
    return found


def test_no_kernel_uses_scratch_memory(kernels):
    for name, (_, _, scratch, _, code) in kernels.items():
        assert scratch == 0 and not re.search(r"\b(scratch|buffer)_(load|store)", code), name


def test_arguments_fit_a_launch(kernels):
    for name, (_, arguments, *_) in kernels.items():
        assert arguments <= 4096, name


def test_a_workgroup_of_1024_lanes_fits_a_cu(kernels):
    """Four waves on each of its four units, which have 512 registers a lane."""
    for name, (registers, _, _, lanes, _) in kernels.items():
        if lanes == 1024:
            assert registers <= 128, name


def test_no_packed_fp32(kernels):
    for name, (*_, code) in kernels.items():
        assert not re.search(r"v_pk_(add|mul|fma)_f32", code), name
