"""Inline assembly of the answers', the orthogonalised step's and the 8-bit products' kernels, checked as that of the other operators of the
head is."""
import tempfile
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

import test_head_isa as isa
import test_isa_hazards as hazards
from paper_1502_03409_amd import build as B

SOURCES = ["logp_f32.hip", "logp_bf16.hip", "muon_f32.hip", "muon_bf16.hip", "q8_f32.hip", "q8_bf16.hip"]


@pytest.fixture(scope="module")
def assembly():
    with tempfile.TemporaryDirectory() as d:
        with ThreadPoolExecutor(max_workers=6) as ex:
            return dict(zip(SOURCES, ex.map(lambda s: hazards._assembly(B.CSRC / s, Path(d) / (s + ".s")), SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_loads_into_lds_carry_their_wait_states(assembly, source):
    isa.test_loads_into_lds_carry_their_wait_states(assembly, source)


@pytest.mark.parametrize("source", SOURCES)
def test_a_barrier_of_the_loads_waits_for_them(assembly, source):
    isa.test_a_barrier_of_the_loads_waits_for_them(assembly, source)


@pytest.mark.parametrize("source", SOURCES)
def test_kernels_have_names_that_both_passes_agree_on(assembly, source):
    """An unnamed type in a kernel's signature is numbered by the host's and the device's pass apart, and its launch finds no kernel."""
    names = [l.split()[1] for l in assembly[source].splitlines() if l.strip().startswith(".amdhsa_kernel")]
    assert len(names) > 5 and not [n for n in names if "$" in n]
