"""Attention over latent rows at the end of the range that its header gives: channels of 2^60, under weights as far above one as they get without a piece being done again."""
import numpy as np
import pytest

import latent_oracle as O
from test_gpu_latent import Side, check_decode, check_resume, decode, resume

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [16, 60, 128])
@pytest.mark.parametrize("rise", [24.0, 32.0])
def test_channels_of_2_to_the_60(heads, rise):
    """Scores rise by 24 nats behind the first tile (16 weights of 2^34.6 sum to 2^38.6, below the 2^40 that a piece is done again for), or by 32 (above)."""
    n, new, lat = 1500, 9, 512
    side = Side(lat, 64, 16, [n, 40])
    rows = side.draw(n + 40, side.w)
    rows[:, :lat] = np.clip(rows[:, :lat], -2, 2) * 2.0 ** 59
    rows[:, lat:] = 0.0
    rows[64:n, lat] = rise
    side.append([n, 40], rows)
    q = side.draw(new + 1, heads, side.w)
    q[..., :lat] *= 2.0 ** -60                                          # (powers of two: exact in bf16)
    q[..., lat] = 25.0                                                  # by the scale of 0.04, one
    check_resume(side, q, [new, 1], 0.04, resume(side, q, [new, 1], 0.04))
    check_decode(side, q[:2], 0.04, decode(side, q[:2], 0.04))
