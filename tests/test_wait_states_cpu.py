"""The library's machine code, as built: distances between instructions that the hardware leaves to the program.  The compiler keeps
them for its own instructions, not within and around inline assembly.

A copy from memory to LDS takes its LDS address from m0, which a scalar instruction must have written one wait state earlier at
least; a DPP instruction reads another lane's register that a vector instruction must have written two earlier; a result of the
matrix unit may be read by other vector instructions as many wait states later as its instruction has passes, and four more."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_1810_09868_amd import binding as B

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


def too_close(listing):
    """(copies to LDS, those whose m0 the instruction before writes) in a disassembly."""
    copies, bad, before = 0, [], ""
    for line in listing.splitlines():
        if re.match(r"[0-9a-f]+ <", line):
            before = ""
            continue
        inst = line.split("//")[0].strip()
        if inst.startswith("global_load_lds") or inst.startswith("buffer_load") and inst.split()[-1] == "lds":
            copies += 1
            if re.match(r"s_\w+ m0,", before):
                bad.append(inst)
        if inst:
            before = inst
    return copies, bad


def test_the_check_itself():
    at = "0000 <kernel>:\n\ts_mov_b32 m0, s3   // 0: 1\n%s\tglobal_load_lds_dwordx4 v[0:1], off   // 4: 2\n"
    assert too_close(at % "") == (1, ["global_load_lds_dwordx4 v[0:1], off"])
    assert too_close(at % "\ts_nop 0\n") == (1, []) == too_close(at % "\ts_mov_b64 exec, s[4:5]\n")
    assert len(too_close("\ts_mov_b32 m0, s3\n\tbuffer_load_dwordx4 v0, s[0:3], s4 offen lds\n")[1]) == 1


def registers(text):
    out = set()
    for lo, hi, one in re.findall(r"\bv\[(\d+):(\d+)\]|\bv(\d+)\b", text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return out


def dpp_too_early(listing):
    """(DPP instructions, those whose first source a vector instruction has written less than two wait states before)."""
    count, bad, before = 0, [], []
    for line in listing.splitlines():
        if re.match(r"[0-9a-f]+ <", line):
            before = []
            continue
        inst = line.split("//")[0].strip()
        if not inst:
            continue
        op, _, args = inst.partition(" ")
        if op.startswith("v_") and re.search(r" (quad_perm:|row_|bound_ctrl|dpp)", inst):
            count, states, source = count + 1, 0, registers(args.split(",")[1])
            for earlier, to in reversed(before[-2:]):
                if states < 2 and to & source:
                    bad.append(inst)
                    break
                states += int(earlier.split()[1], 0) + 1 if earlier.startswith("s_nop") else 1
        to = registers(args.split(",")[0]) if op.startswith("v_") and not op.startswith("v_cmp") else set()
        before = before[-1:] + [(inst, to)]
    return count, bad


def test_the_check_of_dpp_itself():
    at = "\tv_max3_f32 v48, v1, v2, 0   // 0: 1\n%s\tv_max_f32_dpp v3, v48, v48 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n"
    assert len(dpp_too_early(at % "")[1]) == len(dpp_too_early(at % "\ts_nop 0\n")[1]) == len(dpp_too_early(at % "\tv_mov_b32 v9, 0\n")[1]) == 1
    assert dpp_too_early(at % "\ts_nop 1\n") == dpp_too_early(at % "\tv_mov_b32 v9, 0\n\ts_nop 0\n") == (1, [])


PASSES = {"v_mfma_f32_32x32x16_bf16": 8, "v_mfma_f32_32x32x16_f16": 8, "v_mfma_f32_16x16x32_bf16": 4, "v_mfma_f32_16x16x32_f16": 4}


def results_too_early(listing):
    """(vector instructions that read a result of the matrix unit within 16 wait states, those that do too early); what follows a
    branch in the listing is not looked at together with what precedes it."""
    count, bad, before = 0, [], []
    for line in listing.splitlines():
        inst = line.split("//")[0].strip()
        op, _, args = inst.partition(" ")
        if not inst or re.match(r"[0-9a-f]+ <", line) or op.startswith(("s_branch", "s_cbranch", "s_endpgm", "s_setpc")):
            before = [] if inst else before
            continue
        to, _, sources = args.partition(",")
        if op.startswith("v_") and not op.startswith("v_mfma"):
            states, source = 0, registers(sources)
            for earlier, written, passes in reversed(before):
                if source & written:
                    count += passes > 0
                    if 0 < passes and states < passes + 4:
                        bad.append(inst)
                    break
                states += int(earlier.split()[1], 0) + 1 if earlier.startswith("s_nop") else 1
        before = before[-15:] + [(inst, registers(to) if op.startswith("v_") else set(), PASSES.get(op, 0))]
    return count, bad


def test_the_check_of_results_itself():
    at = "\tv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]\n%s\tv_max_f32_e64 v30, v3, 0\n"
    assert len(results_too_early(at % "\ts_nop 10\n")[1]) == 1 and results_too_early(at % "\ts_nop 11\n") == (1, [])
    assert results_too_early(at % "\tv_mov_b32 v3, 0\n") == (0, []) == results_too_early(at % "\ts_cbranch_scc1 5\n")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    lib = shutil.copy(B.LIB_PATH, tmp_path_factory.mktemp("code"))
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True)
    return [subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", code], check=True, capture_output=True, text=True).stdout
            for code in glob.glob(lib + ".*gfx950")]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_no_copy_to_lds_follows_the_write_of_its_address(listings):
    found = [too_close(listing) for listing in listings]
    assert sum(n for n, _ in found) > 1000 and not sum((bad for _, bad in found), [])


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_no_lane_reads_another_lanes_register_too_early(listings):
    found = [dpp_too_early(listing) for listing in listings]
    assert sum(n for n, _ in found) > 100 and not sum((bad for _, bad in found), [])


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_no_result_of_the_matrix_unit_is_read_too_early(listings):
    found = [results_too_early(listing) for listing in listings]
    assert sum(n for n, _ in found) > 1000 and not sum((bad for _, bad in found), [])
