"""xrl_orthogonalise where its symmetric products run in the largest tiles.

Definitions and tolerances are those of test_gpu_orthogonalise."""
import pytest
import torch

import paper_2304_14698_b200 as xrl
from test_gpu_orthogonalise import DTYPES, TOL, define, make, off

pytestmark = pytest.mark.gpu


# Pairs of CTAs on 256 rows take symmetric products of 60 tiles and more: fewer than the 74 pairs that the GPU holds, more than
# those (a pair's second tile), wide and tall, sides that end inside a tile
@pytest.mark.parametrize("dtype,shape", [("bf16", (12, 520, 700)), ("bf16", (12, 700, 520)), ("bf16", (80, 200, 150)), ("bf16", (80, 150, 200)),
                                         ("bf16", (25, 520, 515)), ("bf16", (1, 2900, 2950)), ("bf16", (1, 2950, 2900)),
                                         ("fp32", (12, 520, 700)), ("fp32", (12, 700, 520)), ("fp32", (80, 200, 150)), ("fp32", (80, 150, 200))])
def test_symmetric_products_of_pairs(dtype, shape):
    for kind in ("gradient", "normal"):
        g = make(dtype, *shape, seed=shape[1], kind=kind)
        status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
        got = xrl.xrl_orthogonalise(g, device_status=status)
        assert int(status) == 0
        want = define(g)
        for z in range(shape[0]):
            assert off(got[z], want[z]) <= TOL[dtype], (kind, z)
        assert torch.equal(xrl.xrl_orthogonalise(g), got)
