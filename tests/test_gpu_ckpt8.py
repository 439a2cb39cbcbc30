"""Activation checkpoints in 8 bits: the form itself, bit for bit, and the calls that use it, against 64 bits."""
import pytest
import torch

import kept
from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
TYPES = {"f32": (dk.DK_F32, torch.float32), "bf16": (dk.DK_BF16, torch.bfloat16)}


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    assert dk.dk_device_status(c) == 0
    c.close()


def draw(rows, d, dt, seed=0, spread=8.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + d)
    x = torch.randn((rows, d), generator=g, device="cuda")
    return (x * torch.exp2(spread * torch.randn((rows, d), generator=g, device="cuda"))).to(dt)


def stored(ctx, x, fill=0xAB):
    rows, d = x.shape
    q = dk.dk_ckpt8(rows, d, dk.DK_F32 if x.dtype == torch.float32 else dk.DK_BF16)
    assert dk.dk_ckpt8_bytes(q) == kept.size(rows, d)
    ckpt = torch.full((kept.size(rows, d),), fill, dtype=torch.uint8, device="cuda")
    dk.dk_ckpt8_store(ctx, q, x, ckpt)
    return ckpt


SHAPES = [(1, 1), (3, 31), (5, 32), (2, 33), (7, 60), (4, 100), (9, 34), (196, 512), (1, 16384), (33, 1001), (300, 4096),
          (70001, 64), (16385, 1000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_store_and_load(ctx, rows, d, dtype):
    code, dt = TYPES[dtype]
    x = draw(rows, d, dt)
    ckpt = stored(ctx, x)
    q, b = kept.encode(x)
    got_q, got_b = kept.parts(ckpt, rows, d)
    assert torch.equal(got_b, b) and torch.equal(got_q, q)
    want = kept.values(q, b, d)
    # within half a step, and half a step at most 1/127 of the block's largest
    step = kept.power(b.to(torch.int64) - 127).repeat_interleave(32, dim=1)[:, :d]
    assert bool(((want - x.double()).abs() <= step / 2).all())
    for c, t in TYPES.values():                    # (loaded as either type: the values are bf16 numbers)
        y = torch.full((rows, d), float("nan"), dtype=t, device="cuda")
        dk.dk_ckpt8_load(ctx, dk.dk_ckpt8(rows, d, c), ckpt, y)
        assert torch.equal(y.double(), want)


def test_borders(ctx):
    """Halves, the value that would round to 128, the ends of fp32's range, zeros, infinities and NaN."""
    nan, inf = float("nan"), float("inf")
    top = torch.finfo(torch.float32).max
    rows = [[127.0, 0.5, 1.5, -2.5, 126.5, -0.5], [127.5, 0.5, 1.5, 2.5, 3.0], [127.49999, 0.5], [63.75, 63.7499961853, 1.0],
            [1.0, 1e-30], [0.0, -0.0], [top, -top, 1e38], [2.0 ** -126, 2.0 ** -127, 2.0 ** -130], [1e-45, -1e-45],
            [64 * 2.0 ** -126, 2.0 ** -127, 3 * 2.0 ** -128], [inf, 1.0], [nan, 1.0], [-inf, nan], [2.0 ** -120, -(2.0 ** -121)]]
    x = torch.zeros((len(rows), 70), device="cuda")
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r)
        x[i, 64:66] = torch.tensor([1.0, 0.3])     # (a block beside it that is as it should be)
    q, b = kept.encode(x)
    got = kept.parts(stored(ctx, x), len(rows), 70)
    assert torch.equal(got[1], b) and torch.equal(got[0], q)
    assert b[10:13, 0].tolist() == [255] * 3 and bool((b[:, 2] == b[0, 2]).all())
    y = torch.empty_like(x)
    dk.dk_ckpt8_load(ctx, dk.dk_ckpt8(len(rows), 70, dk.DK_F32), stored(ctx, x), y)
    assert bool(torch.isnan(y[10:13, :32]).all()) and bool(torch.isfinite(y[:, 32:]).all()) and bool(torch.isfinite(y[:10]).all())


@pytest.mark.parametrize("d", [64, 60])
def test_rows_past_32_bits_of_offset(ctx, d):
    """More than 2^31 codes; the first and the last rows are looked at."""
    rows = (1 << 31) // 64 + 1000
    x = torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda")
    for at in (slice(0, 500), slice(rows - 500, rows)):
        x[at] = draw(500, d, torch.bfloat16, seed=at.start)
    ckpt = stored(ctx, x)
    q, b = kept.parts(ckpt, rows, d)
    for at in (slice(0, 500), slice(rows - 500, rows)):
        want = kept.encode(x[at])
        assert torch.equal(q[at], want[0]) and torch.equal(b[at], want[1])
    y = torch.ones_like(x)
    dk.dk_ckpt8_load(ctx, dk.dk_ckpt8(rows, d, dk.DK_BF16), ckpt, y)
    for at in (slice(0, 500), slice(rows - 500, rows)):
        assert torch.equal(y[at].double(), kept.values(*kept.encode(x[at]), d))
    assert not bool(y[500:rows - 500].any())


# ---- group normalisation -------------------------------------------------------------------------------------------
NORMS = [(4, 7, 7, 512, 32), (2, 5, 3, 6, 2), (27, 37, 53, 60, 5), (3, 56, 56, 64, 32), (1, 1, 1, 40, 4), (5, 9, 11, 33, 1),
         (2, 64, 64, 96, 3), (600, 8, 8, 32, 8), (17000, 1, 2, 36, 4)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("n,h,w,c,groups", NORMS)
def test_group_norm(ctx, n, h, w, c, groups, act, dtype):
    """Forward: the bits of the call without a checkpoint and of the store.  Backward: the bits of the call on the
    checkpoint's values as a tensor of their own (tests of that call hold it against 64 bits)."""
    code, dt = TYPES[dtype]
    x, dy = draw(n * h * w, c, dt, spread=0.5), draw(n * h * w, c, dt, seed=1, spread=0.5)
    g = torch.Generator(device="cuda").manual_seed(3)
    gamma, beta = (torch.randn(c, generator=g, device="cuda") for _ in range(2))
    q = dk.dk_norm(n, h, w, c, groups, act, code, 1e-5)
    ctx.ensure_workspace(q)
    y, y8 = torch.empty_like(x), torch.empty_like(x)
    stats, stats8 = (torch.empty((n, groups, 2), device="cuda") for _ in range(2))
    ckpt = torch.full((kept.size(n * h * w, c),), 0x5C, dtype=torch.uint8, device="cuda")
    dk.dk_group_norm_fwd(ctx, q, x, gamma, beta, y, stats)
    dk.dk_group_norm_fwd_ckpt8(ctx, q, x, gamma, beta, y8, stats8, ckpt)
    assert torch.equal(y, y8) and torch.equal(stats, stats8)
    assert torch.equal(ckpt, stored(ctx, x))
    back = torch.empty_like(x)
    dk.dk_ckpt8_load(ctx, dk.dk_ckpt8(n * h * w, c, code), ckpt, back)
    out = [[torch.full_like(x, 9.0), torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")] for _ in range(2)]
    dk.dk_group_norm_bwd(ctx, q, dy, back, gamma, beta, stats, *out[0])
    dk.dk_group_norm_bwd_ckpt8(ctx, q, dy, ckpt, gamma, beta, stats, *out[1])
    for a, b in zip(*out):
        assert torch.equal(a, b)
    dk.dk_group_norm_fwd_ckpt8(ctx, q, x, gamma, beta, x, stats8, ckpt)          # in place: the checkpoint is x's still
    assert torch.equal(x, y) and torch.equal(kept.decode(ckpt, n * h * w, c), back.double())


def test_group_norm_of_nothing(ctx):
    q = dk.dk_norm(0, 3, 3, 40, 4, 1, dk.DK_F32, 1e-5)
    ctx.ensure_workspace(q)
    e, c = torch.empty((0, 3, 3, 40), device="cuda"), torch.ones(40, device="cuda")
    k, s = torch.empty(0, dtype=torch.uint8, device="cuda"), torch.empty(0, device="cuda")
    dk.dk_group_norm_fwd_ckpt8(ctx, q, e, c, c, e, s, k)
    dg, db = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    dk.dk_group_norm_bwd_ckpt8(ctx, q, e, k, c, c, s, e, dg, db)
    assert not bool(dg.any()) and not bool(db.any())


# ---- weight gradient -----------------------------------------------------------------------------------------------
def wgrad_bound(dy, x, dtype):
    """Sums of products, the sum S of their magnitudes: a promotion every 4 stages of 64 rows (fp32: 2) is one rounding of
    2^-24, each of the 4 instructions of a stage and product before it loses at most two units of 2^-23; joins of slices,
    the undone powers of two, `scale` and the compensation are some 8 roundings more.  fp32: dy's terms leave 2^-22 of
    themselves, or of 2^-17 of the output's largest dy."""
    rows = dy.shape[0]
    S = dy.abs().t() @ x.abs()
    stages = -(-rows // 64)
    per = 4 if dtype == "bf16" else 2 * 2
    units = 2.0 * 4 * min(per, stages) + (stages / (4 if dtype == "bf16" else 2) + 8) / 2
    # (a product or sum below fp32's normal range, 2^-126, may be lost at each of the rows' additions)
    tol = S * units * 2.0 ** -23 + rows * 2.0 ** -126
    if dtype == "f32":
        tol = tol + S * 2.0 ** -22 + (dy.abs().amax(dim=0) * 2.0 ** -39)[:, None] * x.abs().sum(dim=0)[None]
        tol = tol + (x.abs().max() * 2.0 ** -39) * dy.abs().sum(dim=0)[:, None]
    return tol


WGRADS = [(1, 1, 1), (1, 16, 8), (3, 33, 5), (64, 512, 1000), (65, 60, 129), (128, 256, 256), (2047, 1001, 1502), (500, 64, 7),
          (4096, 512, 384), (256, 5000, 700), (33000, 40, 24), (1000, 96, 2050), (129, 2048, 4096),
          (4000, 2560, 2560), (3900, 2562, 2500), (70, 33, 4001), (2100, 64, 66000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", WGRADS)
def test_wgrad(ctx, rows, d, out, dtype):
    code, dt = TYPES[dtype]
    x = stored(ctx, draw(rows, d, dt, spread=1.0))
    dy = draw(rows, out, dt, seed=5, spread=2.0)
    xv, dyv = kept.decode(x, rows, d), dy.double()
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW, db = torch.full((out, d), float("nan"), device="cuda"), torch.full((out,), float("nan"), device="cuda")
    scale = 0.75
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, scale, 0.0, dW, db)
    want, tol = dyv.t() @ xv * scale, wgrad_bound(dyv, xv, dtype) * scale
    assert bool(((dW.double() - want).abs() <= tol).all()), float(((dW.double() - want).abs() / tol).max())
    # db: at most rows/(8 parts) + 8 + parts additions in a row; 64 of them and more only where rows are many
    depth = rows / 8 + 8 + 64 if rows < 2048 else rows / 64 + 128
    want_b, tol_b = dyv.sum(dim=0) * scale, dyv.abs().sum(dim=0) * scale * (depth + 2) * 2.0 ** -24
    assert bool(((db.double() - want_b).abs() <= tol_b).all())
    # again on top, and without db
    first, first_b = dW.clone(), db.clone()
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, scale, -2.0, dW, db)
    assert bool(((dW.double() - (want - 2 * first.double())).abs() <= tol + 2.0 ** -23 * (first.double().abs() * 3)).all())
    assert bool(((db.double() - (want_b - 2 * first_b.double())).abs() <= tol_b + 2.0 ** -23 * (first_b.double().abs() * 3)).all())
    again = torch.empty_like(dW)
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, scale, 0.0, again, None)
    assert torch.equal(again, first)


@pytest.mark.parametrize("dtype", TYPES)
def test_wgrad_ranges(ctx, dtype):
    """Outputs whose gradients differ by many powers of two keep their digits; so do blocks of x within the range stated."""
    code, dt = TYPES[dtype]
    rows, d, out = 300, 160, 60
    dy = draw(rows, out, dt, spread=0.5) * torch.exp2(-2.0 * torch.arange(out, device="cuda")).to(dt)
    x = draw(rows, d, dt, seed=9, spread=0.5) * torch.exp2(-6.0 * (torch.arange(d, device="cuda") // 32)).to(dt)
    ckpt = stored(ctx, x)
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW = torch.empty((out, d), device="cuda")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, ckpt, 1.0, 0.0, dW, None)
    xv, dyv = kept.decode(ckpt, rows, d), dy.double()
    assert bool(((dW.double() - dyv.t() @ xv).abs() <= wgrad_bound(dyv, xv, dtype)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("of_dy,of_x,scale", [(-100, 100, 1e-6), (60, 60, 1e-37), (-60, -55, 1e30), (-110, 115, 1.0), (90, -95, 1e-30)])
@pytest.mark.parametrize("rows,d,out", [(300, 160, 60), (256, 2560, 4096), (256, 2562, 4096), (2000, 2560, 2560)])
def test_wgrad_far_from_one(ctx, rows, d, out, of_dy, of_x, scale, dtype):
    """Operands' powers of two and `scale` that lie far apart: where the result is a number, so is what leads to it."""
    code, dt = TYPES[dtype]
    dy, x = draw(rows, out, dt, spread=0.5) * 2.0 ** of_dy, draw(rows, d, dt, seed=3, spread=0.5) * 2.0 ** of_x
    ckpt = stored(ctx, x)
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW = torch.empty((out, d), device="cuda")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, ckpt, scale, 0.0, dW, None)
    xv, dyv = kept.decode(ckpt, rows, d), dy.double()
    want, tol = dyv.t() @ xv * scale, wgrad_bound(dyv, xv, dtype) * scale + 2.0 ** -126
    good = (dW.double() - want).abs() <= tol
    if dtype == "bf16":
        # (bf16 operands enter as they are: where the magnitudes of the products add up to more than fp32's largest number, a
        # part of their sum may be more too, before `scale` makes a number of it)
        good = good | (dyv.abs().t() @ xv.abs() >= 2.0 ** 128)
    assert bool(good.all()), float(((dW.double() - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", TYPES)
def test_wgrad_of_infinities(ctx, dtype):
    """An infinity or a NaN in dy spoils its output's row of dW (and db) alone, one in x its block's columns."""
    code, dt = TYPES[dtype]
    rows, d, out = 100, 96, 40
    dy, x = draw(rows, out, dt, spread=0.5), draw(rows, d, dt, seed=2, spread=0.5)
    dy[7, 3], dy[9, 11], x[50, 40] = float("inf"), float("nan"), float("nan")
    ckpt = stored(ctx, x)
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW, db = torch.empty((out, d), device="cuda"), torch.empty(out, device="cuda")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, ckpt, 1.0, 0.0, dW, db)
    bad = torch.zeros((out, d), dtype=torch.bool, device="cuda")
    bad[3], bad[11], bad[:, 32:64] = True, True, True
    assert torch.equal(~torch.isfinite(dW), bad)
    assert (~torch.isfinite(db)).nonzero().flatten().tolist() == [3, 11]
    dy[7, 3] = dy[9, 11] = 0.0
    xv, dyv = kept.decode(ckpt, rows, d), dy.double()
    xv[:, 32:64] = 0.0
    err = (dW.double() - dyv.t() @ xv).abs()
    assert bool((err[~bad] <= wgrad_bound(dyv, xv, dtype)[~bad]).all())


def test_wgrad_of_nothing(ctx):
    q = dk.dk_wgrad8(0, 33, 20, dk.DK_BF16)
    ctx.ensure_workspace(q)
    dy, x = torch.empty((0, 20), dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    dW, db = torch.randn((20, 33), device="cuda"), torch.randn(20, device="cuda")
    want = 0.5 * dW, 0.5 * db
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.5, dW, db)
    assert torch.equal(dW, want[0]) and torch.equal(db, want[1])
    dW[0, 0] = float("nan")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, dW, db)
    assert not bool(dW.any()) and not bool(db.any())
