"""Tiles of the head's products, walked on the host: the sources' own device functions, compiled for the CPU (host_tiles.hip)."""
import os
import random
import re
import subprocess
from pathlib import Path

import pytest

import paper_1502_03409_amd as lc
from paper_1502_03409_amd import binding as B
from paper_1502_03409_amd import build

TYPES = [lc.LC_F32, lc.LC_BF16]
# (count, rows, cols) whose symmetric products take whole tiles of 256 x 256; on the GPU test_gpu_muon_repeats.py calls them twice
LARGE = [(4, 2048, 4096), (4, 4096, 2048), (5, 2000, 4001), (1, 4500, 5000), (1, 5120, 5120)]


@pytest.fixture(scope="module")
def walked(tmp_path_factory):
    program = tmp_path_factory.mktemp("tiles") / "host_tiles"
    # the runtime of the compiler itself has the conversions of fp16 that a host may lack
    cmd = [build.HIPCC, "-std=c++17", "-O1", "-w", "--cuda-host-only", "--rtlib=compiler-rt", "-I", str(build.CSRC),
           str(Path(__file__).parent / "host_tiles.hip"), "-o", str(program)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([str(program)], capture_output=True, text=True, timeout=300, env=dict(os.environ))
    assert r.returncode == 0, r.stderr[-2000:]
    return [l.split() for l in r.stdout.splitlines()]


def symmetric_layouts(count, rows, cols, dtype):
    """(side, waves) of the launches with symmetric results whose tiles store them themselves."""
    plans = lc.head_plan_query(B.LC_HEAD_MUON, count, rows, cols, dtype)
    tiles = [p for p in plans if p["kernel"].startswith("muon_step (") and p["tparam"][3] in (32, 64, 128, 192, 256) and p["arg"][5] == 1]
    return {(p["tparam"][3], p["block"] // 64) for p in tiles if p["arg"][3] == 1}


def test_each_place_of_a_symmetric_result_has_one_writer(walked):
    rows = [list(map(int, w[1:])) for w in walked if w[0] == "symmetric"]
    assert len(rows) > 60
    for side, waves, planes, n, place, least, most in rows:
        assert (least, most) == (1, 1), f"{n} x {n}, tiles of {side} by {waves} waves, {planes} planes, place {place}: {least} to {most} writers"


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_the_walk_has_all_layouts(walked, dtype):
    """Every tile that a stack's symmetric product is planned with has been walked, and the large stacks do take 256 x 256."""
    have = {(int(w[1]), int(w[2])) for w in walked if w[0] == "symmetric"}
    seen = set()
    for shape in LARGE + [(2, 256, 400), (841, 2048, 128), (2, 8192, 4096), (1, 20011, 1021), (3, 65, 40), (1, 4096, 4096), (9, 2436, 2436)]:
        seen |= symmetric_layouts(*shape, dtype)
    assert seen <= have and {s for s, _ in seen} == {32, 64, 128, 192, 256}
    for shape in LARGE:
        assert (256, 8) in symmetric_layouts(*shape, dtype), shape


def test_loads_of_a_later_part_begin_where_it_does(walked):
    """Of a contraction in parts, for every wave and both matrices of a pair."""
    rows = [list(map(int, w[1:])) for w in walked if w[0] == "start"]
    assert len(rows) == 3 * (4 + 8 + 4 + 4 + 8 + 4 + 8)
    for form, waves, wave, step, moved, moved2, want, inside in rows:
        assert moved == moved2 == want and inside, f"form {form}, wave {wave} of {waves}: step {step} begins {moved} and {moved2} bytes on, not {want}"


def test_short_sides_have_the_tiles_that_they_take():
    """Sides of up to 128 take no tile of more than 128 for their first product, and with one plane an operand, where its two planes make
    it a kernel of its own, there are no others."""
    rng = random.Random(11)
    for dtype in TYPES:
        for _ in range(1500):
            short, long = rng.randrange(1, 129), int(2 ** rng.uniform(0, 20))
            count = min(1 << 24, int(2 ** rng.uniform(0, 24)), max(1, (1 << 34) // (short * long)))
            rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
            plans = lc.head_plan_query(B.LC_HEAD_MUON, count, rows, cols, dtype)
            tiles = {p["tparam"][3] for p in plans if p["kernel"] == "muon_step (A)" and p["arg"][5] == 1 and p["tparam"][3]}
            assert tiles <= {32, 64, 128}, (count, rows, cols, tiles)
    kernels = set(re.findall(rb"gemm_kernelILi4ELi\dELi\dELi(\d+)E\w*?PlaneEpiILi2ELb1EE", build.LIB.read_bytes()))
    assert kernels == {b"64", b"128"}
