"""Expired waits of the products behind the loss and the update, in the kernels that the ordinary shapes of the other
tests do not reach: CTA pairs (256 x 256 tiles), with and without slices of the contraction, and the update's one-kernel
form, whose CTAs meet.  A host-set option makes one producer arm a stage without copying, or one CTA not count at a
meeting; with a short poll limit every wait ends within milliseconds, the status says so, and the next call on the
context, whose counters dk_device_status has cleared, is correct.

The shapes follow from the cost rule of the products on 148 SMs: 2000 x 3000 logits of 1000 features are 96 pair tiles,
9 x 40 of 30000 features one tile in 67 slices; X X^T of 2300 x 2500 is 45 pair tiles on and below the diagonal."""
import contextlib

import pytest
import torch

from paper_2207_00083_b200 import binding as dk
from tests import test_gpu_ortho as ortho
from tests import test_gpu_xent as xent

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    c.close()


@contextlib.contextmanager
def withheld(ctx, n):
    dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 12)
    dk.dk_set_option(ctx, dk.DK_OPT_TEST_WITHHOLD, n)
    try:
        yield
        assert dk.dk_get_option(ctx, dk.DK_OPT_TEST_WITHHOLD) == -1          # the hook switched itself off
        assert dk.dk_device_status(ctx) == dk.DK_ERR_TIMEOUT
        assert dk.dk_device_status(ctx) == 0
    finally:
        dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 22)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("dtype,rows,d,vocab,stage", [("f32", 2000, 1000, 3000, 0), ("f32", 2000, 1000, 3000, 5),
                                                      ("bf16", 3000, 600, 5000, 2), ("f32", 9, 30000, 40, 1),
                                                      ("bf16", 9, 60000, 40, 3)])
def test_loss(ctx, dtype, rows, d, vocab, stage, backward):
    dt, tt = xent.TYPES[dtype]
    h, W, t = xent.draw(rows, d, vocab, tt, seed=30)
    q = dk.dk_xent(rows, d, vocab, dt)
    ctx.ensure_workspace(q)
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dh, dW = torch.empty_like(h), torch.empty_like(W)
    if backward:
        dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
    with withheld(ctx, stage):
        if backward:
            dk.dk_linear_xent_bwd(ctx, q, h, W, t, lse, None, 1.0, dh, dW)
        else:
            dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
    xent.check(ctx, h, W, t, dtype, scale=1.0 / rows)


def check_update(ctx, x, dt):
    got, want = ortho.call(ctx, x, dt), ortho.exact(x)
    for g, w in zip(got, want):
        assert float((g.double() - w).norm()) <= (1e-4 if dt == dk.DK_F32 else 2.0 ** -8) * float(w.norm())
    assert dk.dk_device_status(ctx) == 0


@pytest.mark.parametrize("m,n,stage", [(2300, 2500, 0), (2500, 2300, 4)])
def test_update_by_cta_pairs(ctx, m, n, stage):
    x = ortho.draw(1, m, n, torch.float32, seed=31)
    with withheld(ctx, stage):
        ortho.call(ctx, x, dk.DK_F32)
    check_update(ctx, x, dk.DK_F32)


# one meeting a step, two meetings a step (the first is the norm's), several matrices
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,m,n,meeting", [(1, 64, 576, 0), (1, 64, 576, 1), (1, 576, 64, 5), (1, 128, 3000, 1),
                                           (1, 128, 3000, 2), (3, 100, 900, 4)])
def test_update_whose_ctas_meet(ctx, b, m, n, meeting, dtype):
    dt, tt = ortho.TYPES[dtype]
    x = ortho.draw(b, m, n, tt, seed=32)
    with withheld(ctx, meeting):
        ortho.call(ctx, x, dt)
    check_update(ctx, x, dt)
