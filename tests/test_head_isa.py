"""The supervised head's inline-assembly loads, checked in the compiled assembly as those of the layers are: the compiler's hazard
handling does not look inside a statement, so each that holds a memory instruction has its wait states in front of it, sets m0 from
a scalar register only and takes its base from a pair of scalar registers."""
import re
import tempfile
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

import test_isa_hazards as hazards
from paper_1502_03409_amd import build as B

SOURCES = ["glu_f32.hip", "glu_bf16.hip", "xent_f32.hip", "xent_bf16.hip"]


@pytest.fixture(scope="module")
def assembly():
    with tempfile.TemporaryDirectory() as d:
        with ThreadPoolExecutor(max_workers=4) as ex:
            return dict(zip(SOURCES, ex.map(lambda s: hazards._assembly(B.CSRC / s, Path(d) / (s + ".s")), SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_loads_into_lds_carry_their_wait_states(assembly, source):
    loads = 0
    for _, body in hazards._blocks(assembly[source]):
        mem = [k for k, b in enumerate(body) if b.startswith(("global_", "buffer_", "flat_", "scratch_"))]
        if not mem:
            assert all(b.startswith(("s_waitcnt", "s_barrier", ";")) or not b for b in body), body
            continue
        loads += 1
        assert len(mem) == 1 and "_lds_" in body[mem[0]], body
        assert body[mem[0] - 1] == "s_nop 4" and re.fullmatch(r"s_mov_b32 m0, s\d+", body[0]), body
        assert re.search(r"s\[\d+:\d+\]$", body[mem[0]]), body
    assert loads > 100      # every kernel of the source, with its unrolled loads


@pytest.mark.parametrize("source", SOURCES)
def test_a_barrier_of_the_loads_waits_for_them(assembly, source):
    """Barriers written by hand stand behind a wait in the same statement."""
    barriers = 0
    for _, body in hazards._blocks(assembly[source]):
        for k, b in enumerate(body):
            if b.startswith("s_barrier"):
                barriers += 1
                assert k and body[k - 1].startswith("s_waitcnt"), body
    assert barriers > 10
