"""What the compiler does not count inside inline assembly, in the code that is built from the sources here: one wait state between a
scalar write of m0 and a load to LDS that reads it, five between a vector instruction's write of a scalar and its use as an address."""
import os
import re
import shutil
import subprocess
from pathlib import Path

import pytest

import __graft_entry__ as entry

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def unwaited(assembly):
    """Loads to LDS whose m0 was written by the instruction before, or whose address by one of the five before that are vector ones."""
    found, before, loads, recent = [], "", 0, []
    for line in assembly.splitlines():
        text = line.split(";")[0].strip()
        if not text or text.startswith(".") or text.endswith(":"):
            continue
        if re.match(r"(global|buffer|scratch)_load\w*_lds|buffer_load.*\blds\b", text):
            loads += 1
            if re.match(r"s_\w+ m0\b", before):
                found.append((before, text))
            address = re.search(r"s\[(\d+):(\d+)\]", text)
            for past in recent[-5:] if address else ():
                written = re.match(r"v_\w+ s\[?(\d+)(?::(\d+))?", past)
                if written and int(written[1]) <= int(address[2]) and int(written[2] or written[1]) >= int(address[1]):
                    found.append((past, text))
        before = text
        recent.append(text)
    return loads, found


def test_the_check_sees_a_missing_wait():
    load = "\tglobal_load_lds_dwordx4 v1, s[2:3]\n"
    assert unwaited("\ts_mov_b32 m0, s4\n" + load) == (1, [("s_mov_b32 m0, s4", load.strip())])
    assert unwaited("\ts_add_i32 m0, s4, 16 ; comment\n\ts_nop 0\n" + load) == (1, [])
    assert unwaited("\tv_readfirstlane_b32 s3, v4\n\ts_nop 3\n" + load) == (1, [("v_readfirstlane_b32 s3, v4", load.strip())])
    assert unwaited("\tv_readfirstlane_b32 s4, v4\n\ts_nop 3\n" + load) == (1, [])
    assert unwaited("\tv_readfirstlane_b32 s3, v4\n" + 5 * "\ts_nop 0\n" + load) == (1, [])


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no hipcc")
def test_loads_to_lds_wait_for_m0(tmp_path):
    out = tmp_path / "product.s"
    flags = [f for f in entry.HIPCC_FLAGS if f not in ("-shared",)]
    subprocess.run([HIPCC, *flags, f"-I{entry.ROOT / 'include'}", f"-I{entry.CSRC}", "--cuda-device-only", "-S",
                    str(entry.CSRC / "pv_mx_product.hip"), "-o", str(out)], check=True, capture_output=True)
    loads, found = unwaited(out.read_text())
    assert loads > 0 and not found, (loads, found[:3])
