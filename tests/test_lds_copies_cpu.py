"""The library's machine code, as built: a copy from memory to LDS takes its LDS address from m0, which a scalar instruction must
have written one wait state earlier at least.  The compiler keeps that distance for its own copies, not within inline assembly."""
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


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not available")
def test_no_copy_to_lds_follows_the_write_of_its_address(tmp_path):
    lib = shutil.copy(B.LIB_PATH, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True)
    copies, bad = 0, 0
    for code in glob.glob(lib + ".*gfx950"):
        out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", code], check=True, capture_output=True, text=True).stdout
        c, b = too_close(out)
        copies, bad = copies + c, bad + len(b)
    assert copies > 1000 and bad == 0, (copies, bad)
