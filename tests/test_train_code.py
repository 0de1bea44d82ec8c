"""The built gfx950 code of the operators of a training step's end (csrc/train): wait states of direct loads and no vector
registers spilled to scratch memory. Needs no GPU."""
import os

import pytest

import test_isa_hazards as isa

FOLDER = os.path.join(os.path.dirname(isa.BUILD), "csrc", "train")
SOURCES = sorted(f for f in os.listdir(FOLDER) if f.endswith(".hip"))
DIRECT_LOADS = {"ard_headloss.hip", "ard_muon.hip"}


@pytest.mark.skipif(not all(os.path.exists(t) for t in isa.TOOLS), reason="ROCm LLVM tools not found")
@pytest.mark.parametrize("src", SOURCES)
def test_wait_states_and_registers(tmp_path, src):
    if not os.path.exists(os.path.join(isa.BUILD, src + ".o")):
        pytest.skip("library objects not built")
    n, bad = isa.hazards(isa._disassemble(os.path.join(isa.BUILD, src + ".o"), tmp_path))
    assert (n > 0) == (src in DIRECT_LOADS) and not bad, "\n".join(bad[:10])
    isa.test_no_kernel_spills_registers(tmp_path, src)
