"""What the products that attn_latent.hip writes in assembly rely on (tests/test_latent_asm.py), in the machine code of the built library and along every path: round the
loops' back edges and over branches too, where a listing read from top to bottom ends."""
import pytest

from device_code import OBJDUMP, code_objects, functions, registers

pytestmark = pytest.mark.skipif(OBJDUMP is None, reason="needs llvm-objdump")
PRODUCT = "v_mfma_f32_32x32x16_bf16"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("code") / "image.o")
    found = [f for image in code_objects() if b"latent_merge_kernel" in image for f in functions(image, path) if "13latent_kernel" in f.name]
    assert len(found) == 6 * 3 * 2                                     # widths, columns, decode and chunks
    return found


def products(f):
    return [i for i, c in enumerate(f.code) if c.startswith("v_mfma")]


def all_of(f, i):
    return set().union(set(), *map(registers, f.operands(i)))


def test_operands_are_settled(kernels):
    """No vector instruction writes what a product reads within two states before it."""
    for f in kernels:
        for i in products(f):
            assert f.code[i].startswith(PRODUCT + " ")
            read = set().union(*map(registers, f.operands(i)[1:]))
            for j in f.near(i, 2, forward=False):
                if f.code[j].startswith("v_") and not f.code[j].startswith("v_mfma"):
                    assert not registers(f.operands(j)[0]) & read, (f.name, f.code[j], f.code[i])


def test_results_are_waited_for(kernels):
    """Nothing touches a product's result within 20 states behind it but a product into the same registers."""
    for f in kernels:
        for i in products(f):
            dst = registers(f.operands(i)[0])

            def goes_on(j):
                return f.code[j].startswith("v_mfma") and registers(f.operands(j)[0]) == dst

            for j in f.near(i, 20, forward=True, ends=goes_on):
                touched = set().union(*map(registers, f.operands(j)[1:3])) if goes_on(j) else all_of(f, j)
                assert not dst & touched, (f.name, f.code[i], f.code[j])
