"""A head without its logits, on the CPU: m0 in the gfx950 assembly of its kernels.  Loads to LDS take their place from m0, which is written in
inline assembly; the compiler cannot be told so (the register is reserved), so nothing that it makes by itself may go by m0."""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2512_17570_amd import build as B


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: assembly lines}"""
    out = str(tmp_path_factory.mktemp("asm") / "gs_head.s")
    flags = [f for f in B.FLAGS if f != "-shared"]
    subprocess.run([B.HIPCC, *flags, "--offload-device-only", "-S", "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, os.path.join(B.CSRC, "gs_head.hip"),
                    "-o", out], check=True, capture_output=True, text=True)
    text = open(out).read()
    marks = [(m.start(), m[1]) for m in re.finditer(r"^(_ZN2gs\w+):", text, re.M)]
    ends = [a for a, _ in marks[1:]] + [len(text)]
    found = {name: [l.split(";")[0].strip() for l in text[a:e].split(".section")[0].split("\n")] for (a, name), e in zip(marks, ends)}
    assert len(found) == len(re.findall(r"^\s*\.amdhsa_kernel ", text, re.M))
    return found


def foreign(lines):
    """Instructions that go by m0, named or not, beside the writes and loads of the inline assembly."""
    code = [l for l in lines if l]
    own = set()
    for i, l in enumerate(code):
        if re.match(r"s_add_u32 m0, s\d+, ", l) and code[i + 1].startswith("s_nop") and code[i + 2].startswith("global_load_lds_dwordx4 "):
            own |= {i, i + 2}
    goes_by = r"\bm0\b|_load_lds_|\blds\b|^ds_(gws|ordered|gs_reg|add_gs|sub_gs)|movrel|s_set_gpr_idx|^s_sendmsg|^s_ttrace|^v_interp|gpr_idx"
    return [l for i, l in enumerate(code) if i not in own and re.search(goes_by, l)], len(own) // 2


def test_nothing_else_goes_by_m0(kernels):
    loads = 0
    for name, lines in kernels.items():
        others, own = foreign(lines)
        assert not others, (name, others)
        loads += own
    assert loads > 100


def test_the_reader_finds_other_uses():
    own = ["s_add_u32 m0, s4, 1024", "s_nop 0", "global_load_lds_dwordx4 v1, s[2:3]"]
    assert foreign(own) == ([], 1)
    for other in ("s_mov_b32 m0, s7", "v_readlane_b32 s1, v2, m0", "global_load_lds_dword v1, s[2:3]", "s_sendmsg sendmsg(MSG_INTERRUPT)", "s_add_u32 m0, s4, 1024"):
        assert foreign([*own, other, "s_nop 0", "s_endpgm"])[0] == [other]
