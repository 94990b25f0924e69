"""The requests from memory to LDS that are written as instructions of their own (csrc/gemm8.hip, `request_to_lds`).  Each sets the scalar register m0, which the compiler reserves: it can neither be named among
what they change nor is it kept for anybody, but a use of the compiler's own could come to lie behind one of them.  On the built library: in the kernels that hold such requests m0 is set by them
alone, each for itself, and nothing else reads it."""
import os
import re
import subprocess

import pytest

import paper_1806_00187_amd as A
from tests.test_matrix_products_compiled import OBJDUMP, code_objects, kernels

# instructions that read m0 without naming it, loads to LDS apart
READS_M0 = re.compile(r"(s_sendmsg|s_movrel|v_movrel|s_ttracedata|v_interp|ds_gws|ds_\w+_addtid)")


def strangers(instructions):
    """What in a kernel's code touches m0, but is no request as it is written: set, five wait states, load."""
    found, texts = [], [c.text for c in instructions]
    for i, c in enumerate(instructions):
        to_lds = c.name.startswith(("buffer_load", "global_load_lds")) and re.search(r"\blds\b|_lds_", c.text)
        if to_lds:
            if i < 2 or texts[i - 1] != "s_nop 4" or not re.fullmatch(r"s_mov_b32 m0, s\d+", texts[i - 2]):
                found.append(c.text)
        elif re.fullmatch(r"s_mov_b32 m0, s\d+", c.text):
            if i + 2 >= len(texts) or texts[i + 1] != "s_nop 4" or not re.search(r"^buffer_load_dword(x4)? .*\blds$", texts[i + 2]):
                found.append(c.text)
        elif re.search(r"\bm0\b", c.text) or READS_M0.match(c.name):
            found.append(c.text)
    return found


def test_only_the_requests_to_lds_use_the_register_that_they_set(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    seen = 0
    for n, code in enumerate(code_objects(os.path.join(os.path.dirname(A.__file__), "libnmt.so"))):
        if b"gemm8_kernel" not in code:
            continue
        path = tmp_path / f"{n}.o"
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], check=True, capture_output=True, text=True).stdout
        for name, (instructions, _) in kernels(listing).items():
            if "gemm8_kernel" in name:
                assert strangers(instructions) == [], name
                seen += sum(c.text.endswith(" lds") for c in instructions)
    assert seen


REQUEST = """0000000000000100 <k>:
	s_mov_b32 m0, s5                                           // 000000000100: 00000000
	{0:<58} // 000000000104: 00000000
	buffer_load_dwordx4 v0, s[0:3], 0 offen lds                // 000000000108: 00000000
	{1:<58} // 00000000010C: 00000000
	s_endpgm                                                   // 000000000110: 00000000
"""


@pytest.mark.parametrize("wait,behind,found", [("s_nop 4", "s_nop 0", 0), ("s_nop 3", "s_nop 0", 2), ("s_nop 4", "buffer_load_dword v0, s[0:3], 0 offen lds", 1),
                                               ("s_nop 4", "s_sendmsg sendmsg(MSG_INTERRUPT)", 1), ("s_nop 4", "s_mov_b32 m0, -1", 1), ("s_nop 4", "v_readlane_b32 s4, v1, m0", 1)])
def test_the_check_finds_what_uses_it_too(wait, behind, found):
    (instructions, _), = kernels(REQUEST.format(wait, behind)).values()
    assert len(strangers(instructions)) == found
