"""What gfx950 asks of direct global-to-LDS loads, and the compiler does not see to inside an asm statement (csrc/lds_dma.h): a state between a scalar write of M0 and the
load that takes its LDS address from there.  Looked for in the machine code of the built library, along every path."""
import re

import pytest

from device_code import OBJDUMP, code_objects, functions, registers

pytestmark = pytest.mark.skipif(OBJDUMP is None, reason="needs llvm-objdump")


@pytest.fixture(scope="module")
def direct(tmp_path_factory):
    """Functions with direct loads, and where those are."""
    path, found = str(tmp_path_factory.mktemp("code") / "image.o"), []
    for image in code_objects():
        for f in functions(image, path):
            loads = [i for i, c in enumerate(f.code) if c.startswith("global_load_lds") or (c.startswith("buffer_load") and c.endswith(" lds"))]
            if loads:
                found.append((f, loads))
    assert len(found) >= 12 + 4 and sum(len(loads) for _, loads in found) > 1000
    return found


def test_a_state_between_m0_and_the_load(direct):
    wrong = []
    for f, loads in direct:
        for i in loads:
            wrong += [(f.name, f.code[j], f.code[i]) for j in f.near(i, 1, forward=False) if f.operands(j) and f.operands(j)[0] == "m0"]
    assert not wrong, (len(wrong), wrong[:2])


def scalars_written(f, i):
    """Scalar registers that a vector instruction writes: read lanes, compares, carries."""
    x = f.operands(i)
    dsts = [r for r in map(registers, x[:2]) if r]                     # (a carry or a scaled quotient's flag is the second operand)
    out = {r for d in dsts[:1] for r in d}
    if re.match(r"v_(mad_[ui]64|div_scale|(add|addc|sub|subb|subrev|subbrev)_co)", f.code[i]):
        out |= {r for d in dsts for r in d}
    return {r for r in out if r[0] == "s"}


def test_five_states_between_a_vector_write_of_the_base_and_the_load(direct):
    """... which the compiler keeps for its own loads alone: page ids come by v_readlane, and so do scalars that were spilled to lanes."""
    wrong, based = [], 0
    for f, loads in direct:
        for i in loads:
            base = {r for o in f.operands(i) for r in registers(o) if r[0] == "s"}
            based += bool(base)
            wrong += [(f.name, f.code[j], f.code[i]) for j in f.near(i, 5, forward=False) if f.code[j].startswith("v_") and scalars_written(f, j) & base]
    assert based > 1000 and not wrong, (based, len(wrong), wrong[:3])
