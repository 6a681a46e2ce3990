"""The tile arithmetic spreads 16 pairs of scores over its steps: widths where that leaves pairs out do not compile."""
import os
import shutil
import subprocess

import pytest

from paper_2603_10342_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC) and shutil.which("hipcc") is None, reason="needs hipcc")
SOURCE = """#include "attn_tile32.h"
__global__ void k(float* p)
{
    using namespace ag::tile32;
    f32x16 sc[2] = {}, o[%(d)d / 32] = {};
    float m = 0.f, l = 0.f;
    Weights<%(lo)s> a{}, b{};
    softmax_and_value_product<%(d)d, %(lo)s>(true, true, (const unsigned char*)p, sc, 1.f, m, l, a, b, o);
    p[0] = l + o[0][0];
}
"""


@pytest.mark.parametrize("d,lo,fits", [(64, "false", True), (128, "true", True), (256, "false", True), (96, "false", False), (192, "true", False)])
def test_widths(tmp_path, d, lo, fits):
    src = tmp_path / "w.hip"
    src.write_text(SOURCE % dict(d=d, lo=lo))
    r = subprocess.run([build.HIPCC, *build.FLAGS, "-fsyntax-only", str(src)], capture_output=True, text=True)
    assert (r.returncode == 0) == fits, r.stderr
    assert fits or "every pair of scores" in r.stderr
