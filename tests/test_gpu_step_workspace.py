"""The training-step calls stay inside the workspace that they ask for: the buffer registered here is exactly that
long, and what lies behind it in the same allocation is unchanged after the calls."""
import ctypes

import pytest
import torch

from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
GUARD = 96 << 20

CASES = [
    dk.dk_norm(5, 13, 17, 60, 5, 1, 0, 1e-5), dk.dk_norm(3, 60, 60, 64, 1, 2, 1, 1e-5), dk.dk_norm(300, 1, 1, 4096, 4, 0, 0, 1e-5),
    dk.dk_norm(1, 500, 500, 8, 8, 0, 1, 1e-5),
    dk.dk_xent(1, 1, 1, 0), dk.dk_xent(256, 4096, 1000, 0), dk.dk_xent(64, 512, 1000, 0), dk.dk_xent(300, 100, 5001, 1),
    dk.dk_xent(2000, 77, 30001, 0), dk.dk_xent(5000, 64, 20000, 1), dk.dk_xent(700, 2000, 300, 1), dk.dk_xent(8192, 16, 10, 0),
    dk.dk_ortho(1, 1, 1, 0, 5, 3.4445, -4.775, 2.0315, 1e-7), dk.dk_ortho(1, 1961, 1001, 1, 5, 3.4445, -4.775, 2.0315, 1e-7),
    dk.dk_ortho(3, 512, 4608, 0, 2, 3.4445, -4.775, 2.0315, 1e-7), dk.dk_ortho(2, 257, 3000, 0, 2, 3.4445, -4.775, 2.0315, 1e-7),
    dk.dk_ortho(1, 520, 9000, 0, 1, 3.4445, -4.775, 2.0315, 1e-7), dk.dk_ortho(1, 9000, 300, 1, 2, 3.4445, -4.775, 2.0315, 1e-7),
    dk.dk_ortho(7, 100, 100, 0, 2, 3.4445, -4.775, 2.0315, 1e-7), dk.dk_ortho(1, 1800, 1900, 0, 1, 3.4445, -4.775, 2.0315, 1e-7),
]


def name(q):
    return type(q).__name__ + "_" + "_".join(str(getattr(q, f)) for f, _ in q._fields_[:5])


@pytest.mark.parametrize("q", CASES, ids=name)
def test_guard_behind_the_workspace(q):
    ctx = dk.Context(0)
    need = ctx.step_workspace_bytes(q)
    buf = torch.full((need + GUARD + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    off = (-buf.data_ptr()) % 256
    assert dk.lib().dk_set_workspace(ctx.handle, ctypes.c_void_p(buf.data_ptr() + off), need) == 0
    tt = torch.bfloat16 if q.dtype == dk.DK_BF16 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(tt)

    if isinstance(q, dk.dk_norm):
        x, dy = draw(q.n, q.h, q.w, q.c), draw(q.n, q.h, q.w, q.c)
        gamma, beta = torch.ones(q.c, device="cuda"), torch.zeros(q.c, device="cuda")
        y, stats = torch.empty_like(x), torch.empty((q.n, q.groups, 2), device="cuda")
        dk.dk_group_norm_fwd(ctx, q, x, gamma, beta, y, stats)
        dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, y, gamma.clone(), beta.clone())
        out = [y]
    elif isinstance(q, dk.dk_xent):
        h, W = draw(q.rows, q.d), draw(q.vocab, q.d)
        t = torch.randint(0, q.vocab, (q.rows,), generator=g, device="cuda")
        loss, lse = torch.empty(q.rows, device="cuda"), torch.empty(q.rows, device="cuda")
        dh, dW = torch.empty_like(h), torch.empty_like(W)
        dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
        dk.dk_linear_xent_bwd(ctx, q, h, W, t, lse, None, 1.0, dh, dW)
        out = [loss, lse, dh, dW]
    else:
        x = draw(q.batch, q.m, q.n)
        out = [torch.empty_like(x)]
        dk.dk_orthogonalize(ctx, q, x, 1.0, 0.0, out[0])
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(o).all()) for o in out)
    assert bool((buf[off + need:] == 0xA5).all()) and bool((buf[:off] == 0xA5).all())
    ctx.close()


@pytest.mark.parametrize("rows,d,vocab,dtype", [(1, 2048, 128000, 0), (1, 2047, 9000, 1), (8, 1024, 5000, 0), (4, 6144, 300, 0),
                                                (64, 512, 1000, 0), (9, 30000, 40, 0), (9, 60000, 40, 1), (2000, 77, 30001, 0),
                                                (700, 2000, 300, 1), (5000, 64, 20000, 1)])
def test_scoring_in_its_own_workspace(rows, d, vocab, dtype):
    """The forward call alone, in a workspace of dk_xent_fwd_workspace_bytes: the bits it has in the larger one, nothing
    written behind; the backward call refuses that workspace where it is too small."""
    ctx, q = dk.Context(0), dk.dk_xent(rows, d, vocab, dtype)
    tt = torch.bfloat16 if dtype == dk.DK_BF16 else torch.float32
    g = torch.Generator(device="cuda").manual_seed(2)
    h, W = torch.randn((rows, d), generator=g, device="cuda").to(tt), torch.randn((vocab, d), generator=g, device="cuda").to(tt)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    ctx.ensure_workspace(q)
    want = [torch.empty(rows, device="cuda") for _ in range(2)]
    dk.dk_linear_xent_fwd(ctx, q, h, W, t, *want)
    torch.cuda.synchronize()
    need = ctx.step_workspace_bytes(q, forward=True)
    buf = torch.full((need + GUARD + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    off = (-buf.data_ptr()) % 256
    assert dk.lib().dk_set_workspace(ctx.handle, ctypes.c_void_p(buf.data_ptr() + off), need) == 0
    got = [torch.full((rows,), float("nan"), device="cuda") for _ in range(2)]
    dk.dk_linear_xent_fwd(ctx, q, h, W, t, *got)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bool((buf[off + need:] == 0xA5).all()) and bool((buf[:off] == 0xA5).all())
    if need < ctx.step_workspace_bytes(q):
        with pytest.raises(dk.DkError) as e:
            dk.dk_linear_xent_bwd(ctx, q, h, W, t, got[1], None, 1.0, torch.empty_like(h), torch.empty_like(W))
        assert e.value.status == 4                              # DK_ERR_WORKSPACE
    ctx.close()
