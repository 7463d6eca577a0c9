"""Static checks of the grouped and 8-bit products' machine code (no GPU needed: hipcc cross-compiles): nothing spills vector registers,
no load sits in a per-lane loop, and the K loops are straight-line runs of matrix instructions."""
import os
import re
import subprocess

import pytest

from test_kernel_isa import CSRC, FLAGS, HIPCC, blocks


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    out = tmp_path_factory.mktemp("isa") / "grouped_bf16.s"
    p = subprocess.run([HIPCC, *FLAGS, "-S", "--cuda-device-only", os.path.join(CSRC, "grouped_bf16.hip"), "-o", str(out)],
                       capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    return out.read_text()


def kernels(asm, part):
    for name in re.findall(r"\.name:           (\S+)", asm):
        if part in name:
            start = asm.index("\n" + name + ":")
            yield name, asm[start:asm.index(".Lfunc_end", start)]


def test_no_kernel_spills_vector_registers(asm):
    names = re.findall(r"\.name:           (\S+)", asm)
    spills = re.findall(r"\.vgpr_spill_count:\s+(\d+)", asm)
    assert len(names) == len(spills) > 20
    assert not [n for n, s in zip(names, spills) if s != "0"]


def test_no_load_in_a_per_lane_loop(asm):
    for name, text in kernels(asm, "grouped_"):
        for b in blocks(text):
            if b and b[-1].startswith("s_cbranch_execnz"):
                assert not any(i.startswith(("buffer_load", "global_load")) for i in b), name


@pytest.mark.parametrize("f8,bl", [(1, 0), (1, 1), (0, 0), (0, 1)])
def test_k_loop_of_the_256_kernel(asm, f8, bl):
    """Every K tile's 64 (e4m3) or 128 products of a wave run without a spill, a copy between the register files or a copy out of
    vector memory between them, and the accumulators are tied."""
    (name, text), = kernels(asm, f"grouped_mc_kernelIDF16bLb{f8}ELi{bl}E")
    runs = [b for b in blocks(text) if sum(i.startswith("v_mfma") for i in b) >= 60]
    assert runs, name
    for b in runs:
        at = [k for k, i in enumerate(b) if i.startswith("v_mfma")]
        body = b[at[0]:at[-1] + 1]
        assert not any(i.startswith(("scratch_", "v_accvgpr", "v_writelane")) for i in body)
        for i in body:
            if i.startswith("v_mfma"):
                m = re.match(r"v_mfma\S+\s+(a\[\d+:\d+\]), \S+, \S+, (a\[\d+:\d+\])", i)
                assert m and m.group(1) == m.group(2), "accumulator not tied: " + i
        assert sum(bool(re.match(r"s_waitcnt.*vmcnt", i)) for i in body) <= 2


def test_k_loops_of_the_smaller_tiles(asm):
    """The products of a K tile are one straight-line block with no spill between them."""
    seen = 0
    for name, text in kernels(asm, "grouped_mt_kernelI"):
        f8, bm, bn = (int(x) for x in re.search(r"Lb(\d)ELi\d+ELi\d+ELi(\d+)ELi(\d+)E", name).groups())
        per_tile = (bm // 16) * (bn // 16) * (1 if f8 else 2) // 4   # of a wave
        runs = [b for b in blocks(text) if sum(("f8f6f4" in i) if f8 else i.startswith("v_mfma") for i in b) >= per_tile]
        assert runs, name
        for b in runs:
            at = [k for k, i in enumerate(b) if i.startswith("v_mfma")]
            body = b[at[0]:at[-1] + 1]
            assert not any(i.startswith(("scratch_", "v_accvgpr")) for i in body), name
        seen += 1
    assert seen >= 16
