"""LDS DMAs of the 4-bit attention, in the built gfx950 code: each takes its base from
registers that the scalar instruction right before it, or before the DMAs of the same
base right before it, wrote."""

import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2601_21622_amd as sd
from paper_2601_21622_amd import build as sd_build

from test_isa_dma import OBJDUMP


def unguarded(lines):
    """(DMAs seen, those whose base no instruction before the run of DMAs copies)."""
    seen, found, base = 0, [], None
    for line in lines:
        text = line.split("//")[0].strip()
        if not text or text.endswith(":"):
            continue
        copy = re.match(r"s_mov_b64 (s\[\d+:\d+\]),", text)
        m = re.match(r"global_load_lds_\w+ v\d+, (s\[\d+:\d+\])", text)
        if text.startswith("global_load_lds"):
            seen += 1
            if m is None or m[1] != base:
                found.append(text)
        else:
            base = copy and copy[1]
    return seen, found


def test_the_scan_sees_an_unguarded_load():
    copy, load, more = "\ts_mov_b64 s[4:5], s[8:9]", "\tglobal_load_lds_dwordx4 v54, s[4:5] nt", "\tglobal_load_lds_dwordx4 v54, s[4:5] offset:1024 nt"
    assert unguarded([copy, load, more]) == (2, [])
    assert len(unguarded([copy, load, "\ts_nop 0", more])[1]) == 1
    assert len(unguarded([copy, "\tv_readlane_b32 s4, v1, 0", load, more])[1]) == 2


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_4bit_dmas_copy_their_base(tmp_path):
    sd.library()
    lib = str(tmp_path / "lib.so")
    shutil.copy(sd_build.LIB, lib)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    count = 0
    for o in glob.glob(lib + ".*gfx950*"):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", o], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            if "kv4_attn" in part.split("\n", 1)[0]:
                seen, found = unguarded(part.split("\n")[1:])
                count += seen
                assert not found, f"{part.split(chr(10), 1)[0]}: {len(found)} of {seen}, first {found[0]}"
    assert count > 0
