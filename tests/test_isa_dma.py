"""LDS DMAs of the 8-bit kernels, in the built gfx950 code: each takes its base from
registers that the scalar instruction right before it wrote, so that no vector
instruction (a lane's read, a spilled register's) can have written them within the
five wait states that the load would need, whatever the compiler puts around it."""

import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2601_21622_amd as sd
from paper_2601_21622_amd import build as sd_build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
KERNELS = ("kv8_attn_kernel", "vocab_fp8_kernel")


def unguarded(lines):
    """(DMAs seen, those whose base the instruction before does not copy)."""
    seen, found, before = 0, [], ""
    for line in lines:
        text = line.split("//")[0].strip()
        if not text or text.endswith(":"):
            continue
        m = re.match(r"global_load_lds_\w+ v\d+, (s\[\d+:\d+\])", text)
        if text.startswith("global_load_lds"):
            seen += 1
            if m is None or not before.startswith(f"s_mov_b64 {m[1]},"):
                found.append((before, text))
        before = text
    return seen, found


def test_the_scan_sees_an_unguarded_load():
    load = "\tglobal_load_lds_dwordx4 v54, s[4:5] nt"
    assert unguarded(["\ts_mov_b64 s[4:5], s[8:9]", load]) == (1, [])
    assert len(unguarded(["\ts_nop 0", load])[1]) == 1
    assert len(unguarded(["\ts_mov_b64 s[6:7], s[8:9]", load])[1]) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_8bit_dmas_copy_their_base(tmp_path):
    sd.library()
    lib = str(tmp_path / "lib.so")
    shutil.copy(sd_build.LIB, lib)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    count = dict.fromkeys(KERNELS, 0)
    for o in glob.glob(lib + ".*gfx950*"):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", o], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            name = next((k for k in KERNELS if k in part.split("\n", 1)[0]), None)
            if name:
                seen, found = unguarded(part.split("\n")[1:])
                count[name] += seen
                assert not found, f"{part.split(chr(10), 1)[0]}: {len(found)} of {seen}, first {found[0]}"
    assert all(count.values())
