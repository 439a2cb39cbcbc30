"""Contexts of several threads on one device: each call of one may fall between any two steps of another's, and all give
what they give alone."""
import threading

import pytest
import torch

from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu


def norm(c):
    """Backward sums of c channels: 8*c bytes of shared memory."""
    g = torch.Generator(device="cuda").manual_seed(c)
    x, dy = (torch.randn((1, 3, 3, c), generator=g, device="cuda") for _ in range(2))
    gamma, beta, stats = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda"), torch.ones((1, 1, 2), device="cuda")
    q = dk.dk_norm(1, 3, 3, c, 1, dk.DK_ACT_SILU, dk.DK_F32, 1e-5)
    out = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    return q, lambda ctx: dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, *out), out


def ortho(n):
    """One matrix of n columns: CTAs of 64, 128 or 256 of them, each with its own need of shared memory."""
    x = torch.randn((1, 24, n), generator=torch.Generator(device="cuda").manual_seed(n), device="cuda")
    q = dk.dk_ortho(1, 24, n, dk.DK_F32, 1, 1.5, -0.5, 0.0, 1e-7)
    out = (torch.empty_like(x),)
    return q, lambda ctx: dk.dk_orthogonalize(ctx, q, x, 1.0, 0.0, out[0]), out


@pytest.mark.parametrize("make,sizes", [(norm, (16384, 6000, 12288)), (ortho, (50, 120, 37000))], ids=("norm", "ortho"))
def test_threads_with_a_context_each(make, sizes):
    failures = []

    def work(size):
        i = -1
        try:
            ctx = dk.Context(0)
            q, call, out = make(size)
            ctx.ensure_workspace(q)
            call(ctx)
            torch.cuda.synchronize()
            want = [o.clone() for o in out]
            for i in range(1500):
                call(ctx)
                if i % 50 == 0:
                    torch.cuda.synchronize()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
            ctx.close()
        except Exception as e:  # noqa: BLE001 (reported below, with the size)
            failures.append((size, i, repr(e)))

    threads = [threading.Thread(target=work, args=(s,)) for s in sizes]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures
