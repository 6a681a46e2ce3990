"""Rows that ag_rope_rows would write over each other are refused on the host; rows that it only reads may be the same ones."""
import pytest
import torch

from paper_2603_10342_amd import binding as B
from test_rope_latent_cpu import BAD, rows


def test_rows_of_y_that_overlap():
    for more in (dict(yt=0), dict(yt=64), dict(yh=0), dict(yh=120), dict(yt=0, yh=0), dict(xt=0, yt=0, y=4096, x=4096), dict(yt=120, heads=1)):
        assert rows(total=2, **more) == BAD, more
        assert b"overlap" in B.lib().ag_last_error()
    assert rows(total=0, yt=0) == B.AG_OK and rows(total=0, yh=8) == BAD


@pytest.mark.gpu
def test_one_row_for_all_that_x_repeats():
    rope = B.Rope(torch.tensor([0.01 * i for i in range(16)], dtype=torch.float64, device="cuda"))
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    x, y, want = torch.randn(1, 1, 64, device="cuda").expand(7, 3, 64), torch.empty(7, 3, 64, device="cuda"), torch.empty(7, 3, 64, device="cuda")
    B.ag_rope_rows(rope, x, y, i(5), i(7), i(0, 7), 7)
    B.ag_rope_rows(rope, x.contiguous(), want, i(5), i(7), i(0, 7), 7)
    assert torch.equal(y, want) and not torch.equal(y[0], y[1])
    one = torch.zeros(7, 1, 64, device="cuda")
    B.ag_rope_rows(rope, x[:, :1], one.as_strided((7, 1, 64), (64, 0, 1)), i(5), i(7), i(0, 7), 7)        # a single head's stride is not used
    assert torch.equal(one, want[:, :1])
    for bad in (x, y.as_strided((7, 3, 64), (64, 0, 1)), y.as_strided((7, 3, 64), (0, 64, 1))):
        with pytest.raises(B.AgError, match="overlap"):
            B.ag_rope_rows(rope, x, bad, i(5), i(7), i(0, 7), 7)
