"""Static checks of the machine code of what stands between the layers (no GPU needed: hipcc cross-compiles): nothing spills vector registers, and the
rows' kernels have all of a token's rows on their way before they wait."""
import os
import re
import subprocess

import pytest

from test_kernel_isa import CSRC, FLAGS, HIPCC


def assembly(tmp, name):
    out = tmp / (name + ".s")
    p = subprocess.run([HIPCC, *FLAGS, "-S", "--cuda-device-only", os.path.join(CSRC, name + ".hip"), "-o", str(out)], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    return out.read_text()


@pytest.mark.parametrize("name,count", [("norm", 60), ("route", 100), ("rows", 12)])
def test_no_kernel_spills_vector_registers(name, count, tmp_path):
    asm = assembly(tmp_path, name)
    names = re.findall(r"\.name:           (\S+)", asm)
    spills = re.findall(r"\.vgpr_spill_count:\s+(\d+)", asm)
    assert len(names) == len(spills) > count
    assert not [n for n, s in zip(names, spills) if s != "0"]


def test_rows_are_loaded_ahead_of_their_use_and_stored_past_the_caches(tmp_path):
    asm = assembly(tmp_path, "rows")
    checked = 0
    for name in re.findall(r"\.name:           (\S+)", asm):
        start = asm.index("\n" + name + ":")
        text = asm[start:asm.index(".Lfunc_end", start)]
        assert " nt" in text, name    # (the two kinds of store are not made one)
        m = re.search(r"join_rows_kernelI(?:DF16b|DF16_|f)Li(\d)E", name)
        if m:
            loads = 0
            for line in (l.strip() for l in text.split("\n")):
                if line.startswith("global_load_dwordx4"):
                    loads += 1
                elif line.startswith("s_waitcnt") and "vmcnt(" in line:
                    if loads >= int(m.group(1)):
                        break
                    loads = 0
            assert loads >= int(m.group(1)), name
            checked += 1
    assert checked == 9
