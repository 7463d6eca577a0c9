"""Host-side checks of the tiles that layers over stacks of experts and 8-bit weights run their large products on (no GPU)."""
import os
import subprocess

import numpy as np
import pytest

from paper_2312_03415_amd import binding as rl

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_DIR = os.path.join(HERE, "..", "paper_2312_03415_amd")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "grouped_plan_probe")
    p = subprocess.run([HIPCC, "-std=c++17", "-O1", "--offload-arch=gfx950", os.path.join(HERE, "grouped_plan_probe.cpp"), "-o", exe,
                        "-L" + LIB_DIR, "-lrunlora", "-Wl,-rpath," + os.path.abspath(LIB_DIR)], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]

    def ask(kind, rows):
        text = "".join(kind + " " + " ".join(str(int(v)) for v in tuple(r) + (0,) * (6 - len(r))) + "\n" for r in rows)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.strip().split("\n")
        assert len(out) == len(rows)
        return [[int(v) for v in line.split()] for line in out]
    return ask


def up(a, b):
    return -(-a // b)


def k_tiles(K, fp8):
    return up(K, 128 if fp8 else 64)


def products(count, fp8, seed):
    rng = np.random.default_rng(seed)
    dim = lambda hi: max(16, int(np.exp(rng.uniform(np.log(256), np.log(hi)))) // 16 * 16)
    return [(int(np.exp(rng.uniform(np.log(170), np.log(16384)))), 1, dim(12000), dim(16384), fp8, 0) for _ in range(count)]


@pytest.mark.parametrize("fp8", [0, 1])
def test_few_large_tiles_only_where_their_k_is_split(probe, fp8):
    """256 x 256 tiles, one to a compute unit, that are at most half a round leave half the chip idle unless their K is dealt out; what is dealt out is decided by
    the rule that the kernels have.  One group of rows, so that the count of tiles is known."""
    rows = products(3000, fp8, 7) + [(2100, 1, 2320, 4112, fp8, 0), (1800, 1, 2560, 3584, fp8, 0), (1237, 1, 2064, 5456, fp8, 0), (2560, 1, 2816, 8192, fp8, 0)]
    plans = probe("product", rows)
    tiles = [up(r[0], 256) * up(r[2], 256) for r in rows]
    splits = probe("split", [(t, k_tiles(r[3], fp8)) for t, r in zip(tiles, rows)])
    large = few = joins = 0
    for r, (bm, bn, join), t, (whole, runs, per) in zip(rows, plans, tiles, splits):
        if bm != 256:
            assert join == 0, r
            continue
        large += 1
        assert join == (runs > 1), (r, t)     # the join's room and launch exactly where there is something to join
        joins += join
        if t <= 128:
            few += 1
            assert runs > 1, (r, t)
    assert large > 300 and joins > 20 and (fp8 or few > 20)
    assert [p[0] for p in plans[-4:]] == ([128, 128, 64, 128] if fp8 else [128, 128, 256, 256])


@pytest.mark.parametrize("fp8", [0, 1])
def test_a_tile_is_not_larger_than_a_round_of_the_next_smaller_ones_needs(probe, fp8):
    rows = products(2000, fp8, 9)
    for r, (bm, bn, join) in zip(rows, probe("product", rows)):
        n, _, N, K = r[:4]
        of = lambda m, c: up(n, m) * up(N, c)
        if bm == 128:
            assert of(64, 128) > 512, r
        if bm == 256 and not join:
            assert of(128, 128) > 512, r
        if bm <= 64:
            assert of(64, 128) <= 512, r


@pytest.mark.parametrize("experts,n,N,K,fp8,rows", [
    # uneven experts: what there will be decides, not the most there can be (2000 rows of 4 experts are at most 192 tiles of 256 x 256 and about 160)
    (4, 2000, 4096, 4096, 0, 256), (4, 2000, 4096, 4096, 1, 256), (8, 2000, 4096, 4096, 1, 256), (8, 1000, 4096, 4096, 1, 128),
    (8, 1300, 2304, 4096, 0, 64), (64, 4096, 8192, 2048, 1, 64), (3, 1500, 4992, 4096, 1, 128), (8, 3000, 1024, 8192, 0, 256)])
def test_tiles_of_uneven_experts(probe, experts, n, N, K, fp8, rows):
    assert probe("product", [(n, experts, N, K, fp8, 1)])[0][0] == rows


def test_runs_of_a_split_cover_the_k_tiles_once(probe):
    asks = [(t, nt) for t in range(1, 700, 3) for nt in (1, 40, 54, 63, 64, 65, 86, 128, 129, 172)]
    for (t, nt), (whole, runs, per) in zip(asks, probe("split", asks)):
        left = t - whole
        assert left in (0, t % 256) and (left == 0) == (runs == 1)
        assert runs * per >= nt > (runs - 1) * per
        assert left * runs <= 256          # the sums' room


def test_only_calls_that_may_split_bring_room_for_sums():
    """64 MiB of fp32 sums: where the last round of 256 x 256 tiles may be split, and nowhere else."""
    room = 64 << 20
    ask = lambda n, i, o: rl.runlora_workspace_bytes(rl.FWD1, -1, n, i, o, 16, rl.RL_BF16, rl.RL_FP8_B128)
    small = lambda n, i, o: 2 * n * (i + 128) + 64 * n * 16 + 2 * 16 * o + (1 << 16)   # rows in 8 bits, T and its slices, B turned
    assert ask(2100, 4112, 2320) < small(2100, 4112, 2320)
    whole, split = ask(16384, 11008, 4096), ask(16384, 11008, 4160)    # four rounds of tiles, and four with a quarter of a round
    assert room <= split - whole < room + (1 << 20)


def row_tiles(counts, n, fp8):
    """256-row tiles of the experts' rows and of those behind them; an e4m3 expert's first tile begins on a multiple of four."""
    lo = tiles = 0
    for c in list(counts) + [n - int(sum(counts))]:
        hi = lo + int(c)
        if hi > lo:
            tiles += up(hi - (lo & ~3 if fp8 else lo), 256)
        lo = hi
    return tiles


def test_the_split_cases_split(probe):
    """What test_gpu_experts_split.py runs: the large kernel, with room for sums, and by the kernels' rule a last round that is dealt out."""
    split_cases = pytest.importorskip("test_gpu_experts_split")
    begun = {"Y": set(), "dX": set()}
    for n, experts, i, o, r, kind, side, weights in split_cases.CASES:
        for weight in weights:
            fp8 = int(weight == "fp8")
            K, N = (i, o) if side == "Y" else (o, i)
            assert probe("product", [(n, experts, N, K, fp8, 1)])[0] == [256, 256, 1], (n, i, o, side, weight)
            tiles = row_tiles(split_cases.counts(n, experts, kind), n, fp8) * up(N, 256)
            whole, runs, per = probe("split", [(tiles, k_tiles(K, fp8))])[0]
            assert runs > 1 and whole < tiles, (n, i, o, side, weight, tiles)
            if fp8:
                begun[side].update((k * per, min((k + 1) * per, k_tiles(K, fp8))) for k in range(runs))
    for runs in begun.values():                       # both registers of W's scales, and the change between them inside a run
        assert any(a > 64 for a, b in runs) and any(a < 64 < b for a, b in runs)


def test_the_long_cases_run_on_the_smaller_tiles(probe):
    for n, experts, i, o, r, kind, side, tile in pytest.importorskip("test_gpu_experts_split").LONG:
        K, N = (i, o) if side == "Y" else (o, i)
        assert k_tiles(K, 1) > 64
        if tile:
            assert probe("product", [(n, experts, N, K, 1, 1)])[0][0] == tile, (n, K, N)
        else:
            assert probe("few", [(n, experts, N, K, 1, 1)])[0][0] == 1, (n, K, N)
