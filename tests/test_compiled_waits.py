"""What the compiler does not count inside inline assembly: wait states between a scalar write of m0 and a load to LDS that reads it,
in the code that is built from the sources here."""
import os
import re
import shutil
import subprocess
from pathlib import Path

import pytest

import __graft_entry__ as entry

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def unwaited(assembly):
    """Loads to LDS whose m0 was written by the instruction before."""
    found, before, loads = [], "", 0
    for line in assembly.splitlines():
        text = line.split(";")[0].strip()
        if not text or text.startswith(".") or text.endswith(":"):
            continue
        if re.match(r"(global|buffer|scratch)_load\w*_lds|buffer_load.*\blds\b", text):
            loads += 1
            if re.match(r"s_\w+ m0\b", before):
                found.append((before, text))
        before = text
    return loads, found


def test_the_check_sees_a_missing_wait():
    load = "\tglobal_load_lds_dwordx4 v1, s[2:3]\n"
    assert unwaited("\ts_mov_b32 m0, s4\n" + load) == (1, [("s_mov_b32 m0, s4", load.strip())])
    assert unwaited("\ts_add_i32 m0, s4, 16 ; comment\n\ts_nop 0\n" + load) == (1, [])


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no hipcc")
def test_loads_to_lds_wait_for_m0(tmp_path):
    out = tmp_path / "product.s"
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared",)]
    subprocess.run([HIPCC, *flags, f"-I{entry.ROOT / 'include'}", f"-I{entry.CSRC}", "--cuda-device-only", "-S",
                    str(entry.CSRC / "pv_mx_product.hip"), "-o", str(out)], check=True, capture_output=True)
    loads, found = unwaited(out.read_text())
    assert loads > 0 and not found, (loads, found[:3])
