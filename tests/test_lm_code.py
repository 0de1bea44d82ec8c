"""The built gfx950 code of the language-model operators (csrc/lm): the checks that the layers' sources have, wait states
of direct loads and no vector registers spilled to scratch memory. Needs no GPU."""
import os

import pytest

import test_isa_hazards as isa

SOURCES = ["ard_distill.hip", "ard_glu.hip", "ard_linattn.hip"]


def test_every_source_is_checked():
    folder = os.path.join(os.path.dirname(isa.BUILD), "csrc", "lm")
    assert SOURCES == sorted(os.listdir(folder))


@pytest.mark.skipif(not all(os.path.exists(t) for t in isa.TOOLS), reason="ROCm LLVM tools not found")
@pytest.mark.parametrize("src", SOURCES)
def test_wait_states_and_registers(tmp_path, src):
    if not os.path.exists(os.path.join(isa.BUILD, src + ".o")):
        pytest.skip("library objects not built")
    n, bad = isa.hazards(isa._disassemble(os.path.join(isa.BUILD, src + ".o"), tmp_path))
    assert (n > 0) == (src == "ard_glu.hip") and not bad, "\n".join(bad[:10])
    isa.test_no_kernel_spills_registers(tmp_path, src)
