"""The build's check for vector registers copied while lanes are off (CPU only): where two ways meet, a copy ahead of the
instruction that turns lanes back on leaves the others' values behind."""
import os

import pytest

from paper_2509_01083_amd import build_lib

HEAD = """
0000000000001000 <kernel>:
\tv_and_b32_e32 v98, 15, v0                                  // 000000001000: 26C4008F
\ts_and_b64 exec, s[0:1], s[4:5]                             // 000000001004: 86FE0400
\ts_cbranch_execz 2                                          // 000000001008: BF880002 <kernel+0x14>
\tv_mul_hi_u32 v2, v1, v97                                   // 00000000100C: D2860002 0002C301
"""
TAIL = """\tv_or_b32_e32 v5, 16, v4                                    // 000000001028: 280A0890
\ts_endpgm                                                   // 00000000102C: BF810000
"""


def text(*instructions):
    lines = [f"\t{x:<58} // {0x1014 + 4 * i:012X}: 00000000" for i, x in enumerate(instructions)]
    return HEAD + "\n".join(lines) + "\n" + TAIL


RESTORE = "s_or_b64 exec, exec, s[0:1]"
COPY = "v_accvgpr_write_b32 a200, v98"


@pytest.mark.parametrize("move", [COPY, "v_accvgpr_read_b32 v7, a3", "v_mov_b32_e32 v9, v98", "v_mov_b32_e32 v9, 0x100",
                                  "v_mov_b64_e32 v[2:3], v[4:5]", "scratch_store_dword off, v6, off offset:152",
                                  "scratch_load_dwordx2 v[4:5], off, off offset:8"])
@pytest.mark.parametrize("first", [[], ["s_mov_b32 s10, s29"], ["v_writelane_b32 v255, s39, 17", "s_nop 1"]])
def test_copies_ahead_of_the_restore_are_found(move, first):
    assert build_lib.partial_copies(text=text(*first, move, "s_mov_b64 s[62:63], s[92:93]", RESTORE)) == [f"kernel: {move}"]


def test_a_loops_end_counts_too():
    body = ("s_or_b64 exec, exec, s[0:1]", "v_add_u32_e32 v1, 1, v1", "s_andn2_b64 exec, exec, s[2:3]", "s_cbranch_execnz 65500")
    assert build_lib.partial_copies(text=text(*body, COPY, "s_or_b64 exec, exec, s[2:3]")) == [f"kernel: {COPY}"]


@pytest.mark.parametrize("body", [
    ("v_writelane_b32 v255, s39, 17", RESTORE, COPY),  # behind it: all lanes
    ("v_add_u32_e32 v1, 1, v1", "v_mov_b32_e32 v9, v98", RESTORE),  # a program's own, for the lanes that are on
    (COPY, "s_and_saveexec_b64 s[2:3], vcc"),  # another branch begins: the lanes were all on
    (COPY, "s_branch 4", RESTORE),
])
def test_other_moves_are_not(body):
    assert build_lib.partial_copies(text=text(*body)) == []


def test_the_library_has_none():
    if not os.path.exists(build_lib.LIB):
        build_lib.build()
    bad = build_lib.partial_copies(build_lib.LIB)
    assert not bad, bad[:5]


def test_the_check_sees_the_librarys_branches():
    """The patterns fit what the disassembler prints: symbols, addresses and targets."""
    if not os.path.exists(build_lib.LIB):
        build_lib.build()
    lines = build_lib.device_disassembly(build_lib.LIB).splitlines()
    branches = [ln for ln in lines if "s_cbranch_execz" in ln]
    assert len(branches) > 1000 and all(build_lib._LINE.match(ln).group(3) for ln in branches)
    assert sum(bool(build_lib._SYMBOL.match(ln)) for ln in lines) > 100
