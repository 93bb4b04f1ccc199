"""LDS DMAs of the 4-bit attention, in the built gfx950 code: each takes its base from
registers that the scalar instruction right before it wrote."""

import glob
import os
import re
import shutil
import subprocess

import pytest

import paper_2601_21622_amd as sd
from paper_2601_21622_amd import build as sd_build

from test_isa_dma import OBJDUMP, unguarded


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
