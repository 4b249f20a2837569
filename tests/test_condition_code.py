"""Scalar selects and branches of the built library read a condition that a comparison wrote.

The compiler (22.0, gfx950) has once lowered a 64-bit comparison of uniform numbers, which the scalar unit lacks, to a vector one for the
branch and left the select of the same condition with what a shift had written last: a loop over a kernel's work did not end. Kernels whose
ways through their work compare 64-bit counts have that form, so every build of them is looked at: the library's own code objects, in order."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2606_12950_amd import build

LLVM = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build.HIPCC))), "llvm", "bin")
LINE = re.compile(r"\s+([sv]_\w+)\s*([^/]*)")
USES = re.compile(r"s_(cselect|cmov)_b(32|64)$|s_cbranch_scc[01]$")
# what writes the condition as an answer, what as a carry, and what leaves it
ANSWERS = ("s_cmp", "s_bitcmp", "s_and", "s_or", "s_xor", "s_nand", "s_nor", "s_xnor", "s_not", "s_wqm")
CARRIES = ("s_add_u32", "s_sub_u32", "s_addc_u32", "s_subb_u32")
KEEPS = ("s_mov", "s_cselect", "s_cmov", "s_waitcnt", "s_load", "s_buffer_load", "s_branch", "s_cbranch", "s_barrier", "s_nop", "s_mul", "s_pack",
         "s_setprio", "s_bfm", "s_brev", "s_ff1", "s_flbit", "s_sext", "s_bitset", "s_getpc", "s_setpc", "s_swappc", "s_endpgm", "s_sleep", "s_getreg",
         "s_setreg", "s_trap", "s_sendmsg", "s_memtime", "s_memrealtime", "s_code_end")


def wrong(lines):
    """(kernel, use, what wrote the condition last) where that is neither an answer nor, one instruction before, a carry; and the uses."""
    kernel, last, at, out, uses = None, None, 0, [], 0
    for i, line in enumerate(lines):
        if line.startswith("<"):
            kernel, last = line, None
            continue
        m = LINE.match(line)
        if not m:
            continue
        op = m.group(1)
        if USES.match(op):
            uses += 1
            if last is not None and not last.startswith(ANSWERS) and not (last in CARRIES and at == i - 1 and "cselect" in op):
                out.append((kernel, i, op, last))
        elif op.startswith("s_") and not op.startswith(KEEPS):
            last, at = op, i
    return out, uses


def test_the_form_is_seen():
    before = "s_lshl_b32 s4, s5, 6\nv_cmp_lt_i64_e32 vcc, v[0:1], v[2:3]\n"
    for text, found in ((before + "s_cselect_b32 s6, s7, s8\ns_and_b64 vcc, exec, vcc\ns_cbranch_vccnz 12\n", 1),
                        (before + "s_and_b64 s[2:3], exec, vcc\ns_cselect_b32 s6, s7, s8\n", 0),
                        ("s_cmp_lt_i32 s4, s5\ns_mul_i32 s5, s5, s6\ns_cbranch_scc1 4\n", 0),
                        ("s_add_u32 s4, s5, s6\ns_cselect_b64 s[2:3], -1, 0\n", 0),
                        ("s_add_u32 s4, s5, s6\ns_mov_b32 s9, 0\ns_cselect_b64 s[2:3], -1, 0\n", 1),
                        ("s_cmp_lt_i32 s4, s5\ns_add_i32 s5, s5, s6\ns_cbranch_scc1 4\n", 1)):
        bad, uses = wrong(["<kernel>:"] + ["\t" + l for l in text.splitlines()])
        assert len(bad) == found and uses == 1, text


def code_objects(fatbin):
    """The gfx950 code objects of a library's bundles: a magic, a count, and (offset, size, length of the name, name) of each entry."""
    magic, at = b"__CLANG_OFFLOAD_BUNDLE__", 0
    while (at := fatbin.find(magic, at)) >= 0:
        place = at + len(magic) + 8
        for _ in range(struct.unpack_from("<Q", fatbin, place - 8)[0]):
            offset, size, length = struct.unpack_from("<QQQ", fatbin, place)
            place += 24 + length
            if build.ARCH.encode() in fatbin[place - length:place]:
                yield fatbin[at + offset:at + offset + size]
        at += len(magic)


def test_every_condition_is_a_comparison(tmp_path):
    dump, objcopy = os.path.join(LLVM, "llvm-objdump"), shutil.which("objcopy")
    if not os.path.exists(dump) or not objcopy:
        pytest.skip("needs llvm-objdump and objcopy")
    fat = tmp_path / "fatbin"
    subprocess.run([objcopy, "-O", "binary", "--only-section=.hip_fatbin", build.LIB, str(fat)], check=True)
    objects = list(code_objects(fat.read_bytes()))
    assert len(objects) >= len([s for s in build.SOURCES if "api" not in s])
    seen = 0
    for k, obj in enumerate(objects):
        path = tmp_path / f"{k}.co"
        path.write_bytes(obj)
        text = subprocess.run([dump, "-d", str(path)], check=True, capture_output=True, text=True).stdout
        bad, uses = wrong(re.sub(r"^[0-9a-f]+ (<)", r"\1", l) for l in text.splitlines())
        assert not bad, bad[:4]
        seen += uses
    assert seen > 1000
