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


@pytest.mark.parametrize("rows,d,per,held", [(2200000, 1000, 2200000, True), (2200000, 1001, 7, False), (530000, 4096, 1024, True),
                                             (140000, 16000, 140000, False)])
def test_rows_past_32_bits_of_offset(ctx, rows, d, per, held):
    """More than 2^31 values: the last rows come out as in a call of their own (a row's results are its own).  Sums over rows: of
    ones, with parameters of ones, so that dshift counts the rows exactly; they are below 2^24."""
    dt, tail = torch.bfloat16, 4 * 7 * 1024
    q, few = (dk.dk_block(n, d, p, dk.DK_BLOCK_LAYER, dk.DK_BF16, 1e-5, KEEP, SCALE) for n, p in ((rows, per), (tail, min(per, tail))))
    for p in (q, few):
        ctx.ensure_workspace(p)
    g = torch.Generator(device="cuda").manual_seed(2)
    some = [torch.randn((tail, d), generator=g, device="cuda").to(dt) for _ in range(3)]
    first = rows - tail
    first -= first % per if per <= tail else 0                     # (the rows of a gate together)
    h, u, dh_out = (torch.zeros((rows, d), dtype=dt, device="cuda") for _ in range(3))
    for big, small in zip((h, u, dh_out), some):
        big[first:first + tail] = small
    dn, vec = torch.ones((rows, d), dtype=dt, device="cuda"), torch.ones(d, device="cuda")

    def both(q, rows, h, u, dh_out, dn):
        gate = torch.ones((-(-rows // q.rows_per_gate), d), device="cuda")
        new = lambda: torch.empty((rows, d), dtype=dt, device="cuda")      # noqa: E731
        h_out, n, dh, du, stats = new(), new(), new(), new(), torch.empty((rows, 4), device="cuda")
        size = dk.dk_ckpt8_bytes(dk.dk_ckpt8(rows, d, dk.DK_BF16))
        kh, ku = (torch.empty(size, dtype=torch.uint8, device="cuda") if held else None for _ in range(2))
        dgate, dpost, dpre, dshift = torch.empty_like(gate), torch.empty_like(vec), torch.empty_like(vec), torch.empty_like(vec)
        dk.dk_block_norm_fwd(ctx, q, h, u, gate, vec, vec, vec, h_out, n, stats, kh, ku)
        back, a, b = (dk.dk_block_norm_bwd_ckpt8, kh, ku) if held else (dk.dk_block_norm_bwd, h, u)
        back(ctx, q, dh_out, dn, a, b, gate, vec, vec, stats, dh, du, dgate, dpost, dpre, dshift)
        assert bool((dshift == rows).all())
        return h_out, n, stats, dh, du

    want = both(few, tail, *some, dn[:tail])
    got = both(q, rows, h, u, dh_out, dn)
    for a, b in zip(got, want):
        assert torch.equal(a[first:first + tail], b)


def shifted(t):
    """The same tensor 16 bytes behind a 512-byte boundary."""
    if t is None:
        return None
    skip = 16 // t.element_size()
    return torch.empty(t.numel() + skip, dtype=t.dtype, device="cuda")[skip:].view(t.shape).copy_(t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,gate,per", [(300, 96, "rows", 7), (300, 1030, "channel", 1), (77, 4096, "rows", 1), (301, 1001, "none", 1),
                                             (40, 9000, "rows", 3), (5, 33, "rows", 2)])
def test_tensors_on_any_16_bytes(ctx, rows, d, gate, per, dtype):
    """The same bits wherever the tensors begin."""
    c = Case(rows, d, "layer", gate, per, dtype, shift=True)
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    want = [c.h_out, c.n, c.stats, c.kh, c.ku]
    back = [c.backward(ctx, held) for held in (False, True)]
    for k in ("h", "u", "gate", "post", "pre", "shift", "dh_out", "dn"):
        setattr(c, k, shifted(getattr(c, k)))
    got = [shifted(t) for t in want]
    for t in got:
        t.zero_()
    dk.dk_block_norm_fwd(ctx, c.q, c.h, c.u, c.gate, c.post, c.pre, c.shift, *got)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for held, w in zip((False, True), back):
        out = {k: shifted(t) for k, t in w.items()}
        call, h, u = (dk.dk_block_norm_bwd_ckpt8, got[3], got[4]) if held else (dk.dk_block_norm_bwd, c.h, c.u)
        call(ctx, c.q, c.dh_out, c.dn, h, u, c.gate, c.post, c.pre, got[2], *[None if t is None else t.zero_() for t in out.values()])
        for k in w:
            assert w[k] is None or torch.equal(out[k], w[k]), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("branch", [True, False])
@pytest.mark.parametrize("rows,d", [(700, 35), (300, 38), (500, 1001), (400, 2050), (300, 4096), (40, 5120), (40, 7001), (20, 9000), (7, 16384)])
def test_in_place_whatever_the_rows(ctx, rows, d, branch, dtype):
    """h_out over h and dh over dh_out: the bits of a call with tensors of their own."""
    c = Case(rows, d, "layer", "rows", 3, dtype, branch=branch)
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    h, n = c.h.clone(), torch.empty_like(c.n)
    if branch:
        dk.dk_block_norm_fwd(ctx, c.q, h, c.u, c.gate, c.post, c.pre, c.shift, h, n, None)
        assert torch.equal(h, c.h_out) and torch.equal(n, c.n)
    for held in (False, True):
        want = c.backward(ctx, held)
        got = {k: None if t is None else torch.empty_like(t) for k, t in want.items()}
        got["dh"] = c.dh_out.clone()
        call, h, u = (dk.dk_block_norm_bwd_ckpt8, c.kh, c.ku) if held else (dk.dk_block_norm_bwd, c.h, c.u)
        call(ctx, c.q, got["dh"], c.dn, h, u, c.gate, c.post, c.pre, c.stats, *got.values())
        for k in want:
            assert want[k] is None or torch.equal(got[k], want[k]), k
