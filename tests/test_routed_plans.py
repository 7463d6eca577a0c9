"""Host-side checks of how routing deals out its tokens (no GPU): every call fits the kernels' registers, LDS and counters."""
import os
import subprocess

import numpy as np
import pytest

from paper_2312_03415_amd import binding as rl
from test_experts_plans import HERE, HIPCC, LIB_DIR


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plans") / "route_plan_probe")
    p = subprocess.run([HIPCC, "-std=c++17", "-O1", "--offload-arch=gfx950", os.path.join(HERE, "route_plan_probe.cpp"), "-o", exe,
                        "-L" + LIB_DIR, "-lrunlora", "-Wl,-rpath," + os.path.abspath(LIB_DIR)], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]

    def ask(calls):
        text = "".join(" ".join(str(int(v)) for v in c) + "\n" for c in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return np.array(out.split(), dtype=np.int64).reshape(len(calls), 8)
    return ask


def calls():
    rng = np.random.default_rng(5)
    tokens = [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1024, 1025, 5000, 131072, 131073, 10 ** 6, (1 << 23) - 1]
    for experts in range(1, 1025):
        divisors = [g for g in range(1, 65) if experts % g == 0]
        for top in {1, min(experts, 2), min(experts, 8), min(experts, 15), min(experts, 16), min(experts, 31), min(experts, 32), min(experts, 64)}:
            for groups in divisors:
                yield int(rng.choice(tokens)), experts, top, groups
    for n in tokens:
        for experts in (1, 8, 9, 16, 17, 64, 65, 128, 256, 257, 512, 513, 1024):
            yield n, experts, min(experts, 6), 1


def test_every_call_fits(probe):
    c = np.array(list(calls()))
    lanes, per, waves, each, groups, room, lds, lds_wide = probe(c).T
    n, experts, top, limits = c.T
    assert len(c) > 20000
    assert np.isin(lanes, (8, 16, 32, 64)).all() and np.isin(per, (1, 2, 4, 8, 16)).all()
    assert (lanes * per >= experts).all() and (lanes >= top).all() and (lanes >= limits).all()
    assert ((lanes > top) | (lanes == 64) | (top == experts)).all()        # a lane for the choice's neighbour, or everything is chosen, or 64 lanes
    assert ((lanes != 8) | (per == 1)).all()                               # the kernels that there are
    assert (waves >= 4).all() and (waves <= np.where(per > 8, 8, 16)).all()  # the kernels' launch bounds
    assert (lds_wide <= 65536).all() and (lds <= lds_wide).all()             # what a launch may ask for without further ado
    assert (room >= 4 * experts).all() and (room >= 256).all()
    # keys of all rows in 32 bits, and of one in 64, with groups as far apart as they are laid: up to three lanes' words behind each
    side = 64 // lanes
    assert ((limits == 1) | (room >= (experts + 3 * lanes) * 4 * side)).all() and ((limits == 1) | (room >= (experts + 3 * 64) * 8)).all()
    assert (groups <= 512).all() and (each * groups >= n).all() and (each * (groups - 1) < n).all() and (each < 65536).all()
    assert ((groups == 1) | (each % (waves * side) == 0)).all()
    # the place kernel: eight waves' counts and two tables
    assert ((2 + 8) * experts * 4 <= 65536).all()


def test_group_pitch_stays_inside_its_room():
    """The kernel's layout of groups in LDS, as it works it out: the last key of the last group lies in the room of experts + 3 lanes words."""
    for experts in range(1, 1025):
        for groups in (g for g in range(2, 65) if experts % g == 0):
            for lanes in (8, 16, 32, 64):
                if groups > lanes:
                    continue
                size, q = experts // groups, 1
                while 2 * q * groups <= lanes and q < 16:
                    q *= 2
                pitch = -(-size // (2 * q)) * (2 * q) + q
                assert groups * pitch <= experts + 3 * lanes, (experts, groups, lanes)
                inverse = ((1 << 21) + size - 1) // size
                e = np.arange(1024, dtype=np.int64)
                assert (e * inverse < 1 << 32).all() and (e * inverse >> 21 == e // size).all() and inverse < 1 << 24 and size > 0


def test_workspace_covers_the_plan(probe):
    c = np.array([x for x in calls()][::37])
    lanes, per, waves, each, groups, room, lds, lds_wide = probe(c).T
    for (n, experts, top, _), p, w in zip(c, groups, each):
        need = 0 if p == 1 else p * experts * (1 if w < 256 else 2)
        assert rl.runlora_route_workspace_bytes(int(n), int(experts), int(top)) >= need
