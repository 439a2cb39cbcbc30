"""Block norms where the values that a row does not have, or the rows that a team does not have, could reach those that exist."""
import pytest
import torch

from paper_2207_00083_b200 import binding as dk
from test_gpu_block import Case, KEEP, SCALE, TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    assert dk.dk_device_status(c) == 0
    c.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("branch", [True, False])
@pytest.mark.parametrize("rows,d", [(3, 40), (3, 20), (3, 10), (3, 5), (9473, 40), (9473, 20), (37889, 5), (40, 1000), (3, 5000)])
def test_rows_of_one_large_value(ctx, rows, d, branch, dtype):
    """The last row is one value, 2^100: normalised it is zero and 1/sqrt(eps), 1e10, is finite, but their product, which is what
    a place without a value would have, is not.  Whole numbers of 2^100, so sums and mean are exact (1/d is off by less than
    2^-25 of itself for these d; elsewhere rows of one value may have a variance)."""
    c = Case(rows, d, "layer", "none", 1, dtype, branch=branch)
    c.q = dk.dk_block(rows, d, rows, dk.DK_BLOCK_LAYER, c.code, 1e-20, KEEP, SCALE)
    (c.u if branch else c.h)[-1] = 2.0 ** 100
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    mean, rstd = c.stats[-1, 0 if branch else 2], c.stats[-1, 1 if branch else 3]
    assert float(mean) == 2.0 ** 100 and abs(float(rstd) * 1e-10 - 1) < 1e-5
    assert bool(torch.isfinite(c.n).all())
    for held in (False, True):
        for k, t in c.check_backward(ctx, held).items():
            assert t is None or bool(torch.isfinite(t).all()), (k, held)
