"""The latent attention kernel writes its matrix instructions in assembly (csrc/attn_latent.hip), so that the compiler does not keep the waits around them.  This pins, in
the code that it generates for gfx950, what they rely on: no vector instruction writes a product's operands within two states before it, nothing but a product into the same
accumulator touches a product's result within 20 states behind it (16 passes, three, and one), no spilled register is in a loop of products, and M0 is written by the direct
loads alone."""
import os
import re
import shutil

import pytest

from test_lds_dma_asm import HIPCC, device_asm

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC) and shutil.which("hipcc") is None, reason="needs hipcc")


def registers(operand):
    m = re.match(r"([va])\[(\d+):(\d+)\]$|([va])(\d+)$", operand.strip())
    if not m:
        return set()
    return {(m[1], i) for i in range(int(m[2]), int(m[3]) + 1)} if m[1] else {(m[4], int(m[5]))}


def operands(code):
    parts = code.split(None, 1)
    return [registers(x.split()[0]) for x in parts[1].split(",") if x.split()] if len(parts) > 1 else []


def states(code):
    return int(code.split()[1]) + 1 if code.startswith("s_nop") else 1


@pytest.fixture(scope="module")
def blocks(tmp_path_factory):
    """Instructions in order, with labels."""
    text = device_asm("attn_latent.hip", tmp_path_factory.mktemp("asm"))
    out = []
    for line in text.splitlines():
        code = line.split(";")[0].strip()
        if code and not (code.startswith(".") and not code.endswith(":")):
            out.append(code)
    return out


def test_operands_are_settled_and_results_are_waited_for(blocks):
    products = [i for i, c in enumerate(blocks) if c.startswith("v_mfma")]
    assert len(products) > 1000 and all(blocks[i].startswith("v_mfma_f32_32x32x16_bf16 ") for i in products)
    for i in products:
        dst, a, b = operands(blocks[i])[:3]
        left, j = 2, i - 1
        while left > 0 and j >= 0:
            code = blocks[j]
            if not code.endswith(":"):
                if code.startswith("v_") and not code.startswith("v_mfma"):
                    assert not operands(code)[0] & (a | b), (code, blocks[i])
                left -= states(code)
            j -= 1
        left, j = 20, i + 1
        while left > 0 and j < len(blocks):
            code = blocks[j]
            if code.startswith(("s_branch", "s_endpgm")):
                break
            if not code.endswith(":"):
                if code.startswith("v_mfma") and operands(code)[0] == dst:
                    assert not dst & (operands(code)[1] | operands(code)[2]), (blocks[i], code)
                    break
                assert not dst & set().union(*operands(code), set()), (blocks[i], code)
                left -= states(code)
            j += 1


def test_no_spill_among_products(blocks):
    """Scratch loads would also wait for the tiles on their way."""
    block, found = [], 0
    for code in blocks + ["end:"]:
        if code.endswith(":"):
            n = sum(c.startswith("v_mfma") for c in block)
            if n:
                found += 1
                assert not any(c.startswith("scratch_") for c in block), n
            block = []
        else:
            block.append(code)
    assert found > 100


def test_m0_belongs_to_the_direct_loads_only(blocks):
    loads = [i for i, c in enumerate(blocks) if c.startswith("global_load_lds_dword")]
    assert loads and all(re.match(r"s_mov_b32 m0, ", blocks[i - 1]) for i in loads)
    assert [i for i, c in enumerate(blocks) if re.search(r"\bm0\b", c)] == [i - 1 for i in loads]
