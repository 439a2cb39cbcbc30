"""dk_profile_read counts every kernel that a training-step call launches, whichever way the call goes: compared with what
the CUDA profiling interface saw."""
import pytest
import torch
from torch.profiler import ProfilerActivity, profile

from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
QUINTIC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    c.close()


def check(ctx, call):
    call()
    torch.cuda.synchronize()
    dk.dk_profile_reset(ctx)
    with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    seen = [e.name for e in p.events() if e.device_type == torch.autograd.DeviceType.CUDA and "dk::" in e.name]
    assert seen and dk.dk_profile_read(ctx)["other"][2] == len(seen)


# few rows; small tiles; pair tiles with sliced gradients; sliced logits; several pieces
@pytest.mark.parametrize("dtype", [dk.DK_F32, dk.DK_BF16])
@pytest.mark.parametrize("rows,d,vocab", [(1, 100, 300), (64, 512, 1000), (2000, 1000, 3000), (9, 60000, 40), (2100, 40, 40000)])
def test_loss(ctx, rows, d, vocab, dtype):
    tt = torch.float32 if dtype == dk.DK_F32 else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(1)
    h, W = (torch.randn(s, generator=g, device="cuda").to(tt) for s in ((rows, d), (vocab, d)))
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    q = dk.dk_xent(rows, d, vocab, dtype)
    ctx.ensure_workspace(q)
    loss, lse, dh, dW = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(h), torch.empty_like(W)
    check(ctx, lambda: dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse))
    check(ctx, lambda: dk.dk_linear_xent_bwd(ctx, q, h, W, t, lse, None, 1e-3, dh, dW))


# one kernel; small tiles; pair tiles; sliced X X^T; sliced X; no step
@pytest.mark.parametrize("b,m,n,steps", [(1, 64, 576, 5), (1, 300, 700, 5), (1, 2300, 2500, 3), (1, 130, 60000, 2),
                                         (2, 2000, 1500, 1), (1, 60000, 130, 2), (1, 70, 90, 0)])
def test_update(ctx, b, m, n, steps):
    x = torch.randn((b, m, n), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    q = dk.dk_ortho(b, m, n, dk.DK_F32, steps, *QUINTIC, 1e-7)
    ctx.ensure_workspace(q)
    out = torch.empty_like(x)
    check(ctx, lambda: dk.dk_orthogonalize(ctx, q, x, 1.0, 0.0, out))


@pytest.mark.parametrize("n,h,w,c,groups", [(4, 7, 7, 512, 32), (64, 56, 56, 64, 32), (2, 300, 300, 64, 8)])
def test_normalisation(ctx, n, h, w, c, groups):
    x = torch.randn((n, h, w, c), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    gamma, beta = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    q = dk.dk_norm(n, h, w, c, groups, dk.DK_ACT_SILU, dk.DK_F32, 1e-5)
    ctx.ensure_workspace(q)
    y, stats = torch.empty_like(x), torch.empty((n, groups, 2), device="cuda")
    dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(beta)
    check(ctx, lambda: dk.dk_group_norm_fwd(ctx, q, x, gamma, beta, y, stats))
    check(ctx, lambda: dk.dk_group_norm_bwd(ctx, q, x, x, gamma, beta, stats, y, dgamma, dbeta))
