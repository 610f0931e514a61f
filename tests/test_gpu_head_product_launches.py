"""A product head by head with more blocks of rows than a grid takes: the rows of the second launch."""
import pytest
import torch

import paper_2504_04104_amd as sp
from test_gpu_head_product import near, rnd

pytestmark = pytest.mark.gpu


def test_rows_of_a_second_launch():
    border, n, k = 64 * 65535, 16, 32
    m = border + 70
    x, w = torch.zeros(m, 1, k, dtype=torch.bfloat16, device="cuda"), rnd(2, 1, n, k)
    some = torch.cat([torch.arange(0, 70), torch.arange(border - 70, border + 70)]).cuda()
    x[some] = rnd(1, len(some), 1, k)
    out = torch.full((m + 1, 1, n), 3.0, dtype=torch.bfloat16, device="cuda")
    sp.head_product(x, w, out=out[:m])
    near(out[some], x[some], w)
    assert (out[m] == 3).all()
    out[some] = 0
    assert not out[:m].any()
