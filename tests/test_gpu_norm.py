"""Group normalisation with activation against the formula in 64 bits: sizes and values where it can go wrong.

Tolerances.  A value z = (x - mean)*rstd*gamma + beta formed in fp32 is off by a few roundings of its terms: each is at
most max|x|*rstd*|gamma|, |z| or |beta|, the mean's own error (sums about a pivot, joined pairwise) is below 8 ulp of
max|x|, exp adds |z| ulp.  ULPS = 64 roundings of 2^-24 of the sum of those magnitudes bound it; a bf16 result adds
half a unit of its 8 bits (2^-9 of the value, 2^-8 taken).  The sums of the backward pass run over at most a few
thousand terms per thread and are compared with the sum of the terms' magnitudes."""
import math

import pytest
import torch

from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
EPS = 1e-5
ULPS = 64 * 2.0 ** -24
ACTS = {"none": dk.DK_ACT_NONE, "relu": dk.DK_ACT_RELU, "silu": dk.DK_ACT_SILU}
TYPES = {"f32": (dk.DK_F32, torch.float32), "bf16": (dk.DK_BF16, torch.bfloat16)}


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    c.close()


def draw(n, h, w, c, dtype, seed=1, shift=0.0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, h, w, c), generator=g, device="cuda") * spread + shift
    gamma = 1 + 0.2 * torch.randn(c, generator=g, device="cuda")
    beta = 0.2 * torch.randn(c, generator=g, device="cuda")
    dy = torch.randn((n, h, w, c), generator=g, device="cuda")
    return x.to(dtype), gamma, beta, dy.to(dtype)


def forward64(x, gamma, beta, groups, act, eps=EPS):
    n, h, w, c = x.shape
    v = x.double().reshape(n, h * w, groups, c // groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(((v - mean) ** 2).mean(dim=(1, 3), keepdim=True) + eps)
    z = ((v - mean) * rstd).reshape(x.shape) * gamma.double() + beta.double()
    y = z if act == "none" else torch.relu(z) if act == "relu" else z * torch.sigmoid(z)
    return y, z, mean.reshape(n, groups), rstd.reshape(n, groups)


def backward64(dy, x, gamma, beta, groups, act, mean, rstd):
    n, h, w, c = x.shape
    shape = (n, h * w, groups, c // groups)
    xh = (x.double().reshape(shape) - mean.reshape(n, 1, groups, 1)) * rstd.reshape(n, 1, groups, 1)
    z = xh.reshape(x.shape) * gamma.double() + beta.double()
    s = torch.sigmoid(z)
    slope = torch.ones_like(z) if act == "none" else (z > 0).double() if act == "relu" else s * (1 + z * (1 - s))
    d = dy.double() * slope
    xhf = xh.reshape(x.shape)
    q = (d * gamma.double()).reshape(shape)
    dx = rstd.reshape(n, 1, groups, 1) * (q - q.mean(dim=(1, 3), keepdim=True)
                                          - xh * (q * xh).mean(dim=(1, 3), keepdim=True))
    return dx.reshape(x.shape), (d * xhf).sum(dim=(0, 1, 2)), d.sum(dim=(0, 1, 2)), d, xhf


def run_fwd(ctx, x, gamma, beta, groups, act, dt, eps=EPS):
    n, h, w, c = x.shape
    q = dk.dk_norm(n, h, w, c, groups, ACTS[act], dt, eps)
    ctx.ensure_workspace(q)
    y = torch.full_like(x, float("nan"))
    stats = torch.full((n, groups, 2), float("nan"), device="cuda")
    dk.dk_group_norm_fwd(ctx, q, x, gamma, beta, y, stats)
    return q, y, stats


SHAPES = [  # n, h, w, c, groups
    (1, 1, 1, 1, 1), (2, 1, 1, 8, 2), (3, 1, 1, 4100, 4), (4, 7, 7, 512, 32), (2, 5, 3, 7, 7), (3, 9, 11, 60, 5),
    (2, 33, 17, 6, 3), (1, 64, 64, 64, 1), (5, 13, 13, 96, 32), (2, 112, 112, 16, 4), (1, 3, 5, 2048, 1),
    (129, 4, 4, 24, 8), (2, 2, 2, 16384, 64), (1, 300, 300, 1, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
def test_forward(ctx, n, h, w, c, groups, act, dtype):
    dt, tt = TYPES[dtype]
    x, gamma, beta, _ = draw(n, h, w, c, tt, shift=0.5)
    _, y, stats = run_fwd(ctx, x, gamma, beta, groups, act, dt)
    want, z, mean, rstd = forward64(x, gamma, beta, groups, act)
    amp = float(x.double().abs().max())
    # a group of equal (or single) values has variance 0: rstd = 1/sqrt(eps) amplifies what is left of x - mean
    scale = 1 + amp * float(rstd.max()) * float(gamma.abs().max()) + float(z.abs().max()) + float(beta.abs().max())
    assert float((stats[..., 0].double() - mean).abs().max()) <= ULPS * amp
    assert float(((stats[..., 1].double() - rstd) / rstd).abs().max()) <= ULPS * (1 + amp * float(rstd.max()))
    bound = ULPS * scale + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0)
    assert bool(((y.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
def test_backward(ctx, n, h, w, c, groups, act, dtype):
    dt, tt = TYPES[dtype]
    x, gamma, beta, dy = draw(n, h, w, c, tt, seed=2, shift=0.5)
    q = dk.dk_norm(n, h, w, c, groups, ACTS[act], dt, EPS)
    ctx.ensure_workspace(q)
    _, _, mean, rstd = forward64(x, gamma, beta, groups, act)
    stats = torch.stack((mean, rstd), dim=-1).float().contiguous()
    mean, rstd = stats[..., 0].double(), stats[..., 1].double()
    if act == "relu":       # no value within reach of the kink: both sides must take the same decision
        z = ((x.double().reshape(n, h * w, groups, -1) - mean.reshape(n, 1, groups, 1))
             * rstd.reshape(n, 1, groups, 1)).reshape(x.shape) * gamma.double() + beta.double()
        dy = torch.where(z.abs() < 1e-3, torch.zeros_like(dy), dy)
    dx = torch.full_like(x, float("nan"))
    dgamma, dbeta = torch.full((c,), float("nan"), device="cuda"), torch.full((c,), float("nan"), device="cuda")
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dgamma, dbeta)
    want, wg, wb, d, xh = backward64(dy, x, gamma, beta, groups, act, mean, rstd)
    xm = float(xh.abs().max())
    zmax = 1 + xm * float(gamma.abs().max()) + float(beta.abs().max())
    err_xh = float(x.double().abs().max()) * float(rstd.max())          # xhat is off by ulps of this
    scale = float(rstd.max()) * float(dy.double().abs().max()) * (1 + xm * xm) * (zmax + err_xh) * 2
    bound = ULPS * scale + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0)
    assert bool(((dx.double() - want).abs() <= bound).all())
    terms = dy.double().abs().sum(dim=(0, 1, 2))
    assert bool(((dgamma.double() - wg).abs() <= ULPS * (terms * (xm + err_xh) * zmax + 1e-6)).all())
    assert bool(((dbeta.double() - wb).abs() <= ULPS * (terms * (zmax + err_xh) + 1e-6)).all())
    # the order of every sum is fixed: the same call gives the same bits
    dx2, dg2, db2 = torch.empty_like(dx), torch.empty_like(dgamma), torch.empty_like(dbeta)
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx2, dg2, db2)
    assert torch.equal(dx, dx2) and torch.equal(dgamma, dg2) and torch.equal(dbeta, db2)


@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradient_against_differences(ctx, act):
    """<dx, v>, <dgamma, u> and <dbeta, u> against central differences of sum(y*dy) formed in 64 bits.  The difference
    at step 1e-4 is off by ~1e-8 (third derivatives of order one), the gradient by ~1e-6 (fp32): 1e-5 of the terms."""
    n, h, w, c, groups = 3, 6, 5, 24, 4
    x, gamma, beta, dy = draw(n, h, w, c, torch.float32, seed=5)
    q, _, stats = run_fwd(ctx, x, gamma, beta, groups, act, dk.DK_F32)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dgamma, dbeta)
    t = 1e-4
    g = torch.Generator(device="cuda").manual_seed(9)
    for which, grad in (("x", dx), ("gamma", dgamma), ("beta", dbeta)):
        v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
        vals = []
        for s in (t, -t):
            a = {"x": x.double(), "gamma": gamma.double(), "beta": beta.double()}
            a[which] = a[which] + s * v
            y, _, _, _ = forward64(a["x"], a["gamma"], a["beta"], groups, act)
            vals.append(float((y * dy.double()).sum()))
        diff = (vals[0] - vals[1]) / (2 * t)
        got = float((grad.double() * v).sum())
        assert abs(got - diff) <= 1e-5 * float((grad.double() * v).abs().sum())


@pytest.mark.parametrize("shift,spread", [(1e4, 1.0), (-3e5, 10.0), (1e-12, 1e-12), (0.0, 1e15)])
def test_statistics_far_from_zero(ctx, shift, spread):
    """The variance does not cancel: x - mean is formed before it is squared.  A value near `shift` carries ulps of it
    into x - mean, nothing more (64 of them, against the spread)."""
    x, gamma, beta, _ = draw(4, 20, 20, 32, torch.float32, seed=3, shift=shift, spread=spread)
    _, y, stats = run_fwd(ctx, x, gamma, beta, 8, "none", dk.DK_F32, eps=0.0)
    want, z, mean, rstd = forward64(x, gamma, beta, 8, "none", eps=0.0)
    rel = ULPS * (1 + abs(shift) / spread)
    assert float(((stats[..., 1].double() - rstd) / rstd).abs().max()) <= rel
    assert float((y.double() - want).abs().max()) <= rel * 8


def test_outlier_first_value(ctx):
    """The first value a thread sees is its pivot; an outlier there costs at most the bits of the values it covers."""
    x, gamma, beta, _ = draw(1, 64, 64, 8, torch.float32, seed=4)
    x[0, 0, 0, 0] = 1e4
    _, _, stats = run_fwd(ctx, x, gamma, beta, 1, "none", dk.DK_F32)
    _, _, mean, rstd = forward64(x, gamma, beta, 1, "none")
    assert float(((stats[..., 1].double() - rstd) / rstd).abs().max()) <= 512 * 2.0 ** -24
    assert float((stats[..., 0].double() - mean).abs().max()) <= ULPS * 1e4 / 100


def test_constant_input(ctx):
    x = torch.full((2, 8, 8, 16), 3.25, device="cuda")
    gamma, beta = torch.ones(16, device="cuda"), torch.linspace(-1, 1, 16, device="cuda")
    _, y, stats = run_fwd(ctx, x, gamma, beta, 4, "relu", dk.DK_F32)
    assert torch.equal(y, torch.relu(beta).expand_as(y).contiguous())
    assert torch.allclose(stats[..., 1], torch.full_like(stats[..., 1], 1 / math.sqrt(EPS)))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_values_stay_in_their_group(ctx, bad):
    x, gamma, beta, dy = draw(3, 6, 6, 32, torch.float32, seed=6)
    clean = run_fwd(ctx, x, gamma, beta, 4, "silu", dk.DK_F32)[1]
    x2 = x.clone()
    x2[1, 2, 3, 9] = bad                                   # group 1 of sample 1
    q, y, stats = run_fwd(ctx, x2, gamma, beta, 4, "silu", dk.DK_F32)
    other = torch.ones_like(x, dtype=torch.bool)
    other[1, :, :, 8:16] = False
    assert torch.equal(y[other], clean[other])
    assert bool(torch.isnan(y[1, :, :, 8:16]).all())
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dk.dk_group_norm_bwd(ctx, q, dy, x2, gamma, beta, stats, dx, dg, db)
    assert bool(torch.isfinite(dx[other]).all()) and bool(torch.isnan(dx[1, :, :, 8:16]).all())
    assert bool(torch.isfinite(db[:8]).all()) and bool(torch.isfinite(dg[16:]).all())


def test_large_negative_activation_input(ctx):
    """silu far on the negative side: exp overflows to infinity, the value is -0, the slope 0, never a NaN."""
    x, gamma, beta, dy = draw(1, 8, 8, 8, torch.float32, seed=7)
    gamma = gamma * 300
    q, y, stats = run_fwd(ctx, x, gamma, beta, 1, "silu", dk.DK_F32)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dg, db)
    assert all(bool(torch.isfinite(t).all()) for t in (y, dx, dg, db))


def test_no_samples(ctx):
    q = dk.dk_norm(0, 4, 4, 8, 2, dk.DK_ACT_RELU, dk.DK_F32, EPS)
    ctx.ensure_workspace(q)
    gamma, beta = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    e, st = torch.empty((0, 4, 4, 8), device="cuda"), torch.empty((0, 2, 2), device="cuda")
    dk.dk_group_norm_fwd(ctx, q, e, gamma, beta, e, st)
    dg, db = torch.full((8,), 7.0, device="cuda"), torch.full((8,), 7.0, device="cuda")
    dk.dk_group_norm_bwd(ctx, q, e, e, gamma, beta, st, e, dg, db)
    assert float(dg.abs().max()) == 0 and float(db.abs().max()) == 0


def test_offsets_past_32_bits(ctx):
    """More than 2^31 elements: the last samples are those that a 32-bit offset would miss."""
    n, h, w, c, groups = 44, 224, 224, 1000, 8
    assert n * h * w * c > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn((n, h, w, c), generator=g, device="cuda", dtype=torch.bfloat16)
    gamma, beta = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    q, y, stats = run_fwd(ctx, x, gamma, beta, groups, "none", dk.DK_BF16)
    want, _, mean, rstd = forward64(x[-1:], gamma, beta, groups, "none")
    assert float((y[-1:].double() - want).abs().max()) <= 2.0 ** -8 * 8
    dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    dk.dk_group_norm_bwd(ctx, q, y, x, gamma, beta, stats, dx, dg, db)
    want, _, _, _, _ = backward64(y[-1:], x[-1:], gamma, beta, groups, "none", stats[-1:, :, 0].double(),
                                  stats[-1:, :, 1].double())
    assert float((dx[-1:].double() - want).abs().max()) <= 2.0 ** -8 * 8


def test_in_a_graph(ctx):
    """Captured and replayed on other values: nothing but the launches is kept."""
    for shape, groups in (((2, 7, 7, 64), 8), ((6, 90, 90, 64), 16)):
        x, gamma, beta, dy = draw(*shape, torch.float32, seed=11)
        q, y, stats = run_fwd(ctx, x, gamma, beta, groups, "silu", dk.DK_F32)
        dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
        dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dg, db)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dk.dk_group_norm_fwd(ctx, q, x, gamma, beta, y, stats)
            dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dg, db)
        x.copy_(draw(*shape, torch.float32, seed=12)[0])
        graph.replay()
        torch.cuda.synchronize()
        _, y2, stats2 = run_fwd(ctx, x, gamma, beta, groups, "silu", dk.DK_F32)
        dx2, dg2, db2 = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
        dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats2, dx2, dg2, db2)
        assert all(torch.equal(a, b) for a, b in ((y, y2), (stats, stats2), (dx, dx2), (dg, dg2), (db, db2)))


def test_more_samples_than_counters(ctx):
    """Samples in slabs, more of them than the context has counters for."""
    x, gamma, beta, dy = draw(17000, 3, 3, 2048, torch.bfloat16, seed=13)
    q, y, stats = run_fwd(ctx, x, gamma, beta, 1, "none", dk.DK_BF16)
    want, _, mean, rstd = forward64(x[-3:], gamma, beta, 1, "none")
    assert float((y[-3:].double() - want).abs().max()) <= 2.0 ** -8 * 8
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dg, db)
    total = dy.double().sum(dim=(0, 1, 2))
    assert float((db.double() - total).abs().max()) <= 64 * 2.0 ** -24 * float(dy.double().abs().sum(dim=(0, 1, 2)).max())
    want = backward64(dy[-3:], x[-3:], gamma, beta, 1, "none", stats[-3:, :, 0].double(), stats[-3:, :, 1].double())[0]
    assert float((dx[-3:].double() - want).abs().max()) <= 2.0 ** -8 * 8 * float(gamma.abs().max())


def test_another_stream(ctx):
    x, gamma, beta, _ = draw(2, 30, 30, 64, torch.float32, seed=10)
    want = run_fwd(ctx, x, gamma, beta, 8, "silu", dk.DK_F32)[1]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = run_fwd(ctx, x, gamma, beta, 8, "silu", dk.DK_F32)[1]
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals(ctx):
    x, gamma, beta, _ = draw(2, 4, 4, 8, torch.float32)
    y, stats = torch.empty_like(x), torch.empty((2, 2, 2), device="cuda")
    q = dk.dk_norm(2, 4, 4, 8, 2, dk.DK_ACT_RELU, dk.DK_F32, EPS)
    with pytest.raises(ValueError):
        dk.dk_group_norm_fwd(ctx, q, x.to(torch.bfloat16), gamma, beta, y, stats)
    with pytest.raises(ValueError):
        dk.dk_group_norm_fwd(ctx, q, x.transpose(1, 3), gamma, beta, y, stats)
    with pytest.raises(ValueError):
        dk.dk_group_norm_fwd(ctx, q, x, gamma[:4], beta, y, stats)
    fresh = dk.Context(0)
    with pytest.raises(dk.DkError) as e:
        dk.dk_group_norm_fwd(fresh, q, x, gamma, beta, y, stats)
    assert e.value.status == 4                                  # DK_ERR_WORKSPACE
    fresh.close()
    ctx.ensure_workspace(q)
    with pytest.raises(dk.DkError) as e:                        # misaligned
        dk.dk_group_norm_fwd(ctx, dk.dk_norm(1, 4, 4, 8, 2, 1, dk.DK_F32, EPS), x.reshape(-1)[1:129], gamma, beta,
                             y.reshape(-1)[:128], stats.reshape(-1)[:4])
    assert e.value.status == 1
    assert bool(torch.isfinite(x).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 6, 5, 256, 8), (2, 60, 60, 256, 8), (3, 9, 7, 60, 5), (40, 30, 30, 35, 7)])
def test_relu_mask_at_the_kink(ctx, n, h, w, c, groups, dtype):
    """Each channel's beta puts the value of one element within a rounding of the kink.  With dy = 1, dbeta counts the
    active elements of a channel (small integers: exact); it has to count those that the forward call let through, and dx
    has to take the same decision (the group sums being what they are, dx + rstd*(m0 + xhat*m1) is rstd*gamma where
    active and 0 elsewhere: half of that separates the two)."""
    dt, tt = TYPES[dtype]
    x, gamma, beta, _ = draw(n, h, w, c, tt, seed=21)
    q, y, stats = run_fwd(ctx, x, gamma, beta, groups, "relu", dt)
    mean, rstd = (stats[0, :, i].repeat_interleave(c // groups) for i in (0, 1))
    beta = -((x[0, 0, 0].float() - mean) * (gamma * rstd))
    q, y, stats = run_fwd(ctx, x, gamma, beta, groups, "relu", dt)
    dy, dx, dg, db = torch.ones_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dg, db)
    active = y > 0
    assert torch.equal(db.double(), active.sum(dim=(0, 1, 2)).double())
    shape = (n, h * w, groups, c // groups)
    m, r = stats[..., 0].double()[:, None, :, None], stats[..., 1].double()[:, None, :, None]
    xh = (x.double().reshape(shape) - m) * r
    qv = (active.double() * gamma.double()).reshape(shape)
    back = dx.double().reshape(shape) + r * (qv.mean(dim=(1, 3), keepdim=True)
                                             + xh * (qv * xh).mean(dim=(1, 3), keepdim=True))
    assert torch.equal((back > 0.5 * r * gamma.double().reshape(groups, -1)).reshape(x.shape), active)


def test_pixels_up_to_two_to_the_31(ctx):
    """One channel of 2^31 - 4096 pixels, the most: the last slab's index with a step on top stays in 32 bits.  Mean and
    variance are joined over some 750 sums one after the other, half a unit each, the counts likewise: below 448 units of
    2^-24 (64 times 1 + |x|/spread) together; values and gradients are bf16."""
    pix, step = 2 ** 31 - 4096, 1 << 27
    g = torch.Generator(device="cuda").manual_seed(22)
    x, dy = (torch.empty((1, 1, pix, 1), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        for i in range(0, pix, step):
            v = t.view(-1)[i:i + step]
            v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
    gamma, beta = torch.full((1,), 1.5, device="cuda"), torch.full((1,), 0.25, device="cuda")
    q, y, stats = run_fwd(ctx, x, gamma, beta, 1, "none", dk.DK_BF16)

    def total(f):
        return sum(float(f(x.view(-1)[i:i + step].double(), dy.view(-1)[i:i + step].double()).sum())
                   for i in range(0, pix, step))

    mean = total(lambda a, d: a) / pix
    rstd = (total(lambda a, d: (a - mean) ** 2) / pix + EPS) ** -0.5
    amp = float(x.view(-1)[:step].float().abs().max())
    assert abs(float(stats[0, 0, 0]) - mean) <= ULPS * amp
    assert abs(float(stats[0, 0, 1]) / rstd - 1) <= ULPS * (1 + amp * rstd)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    dk.dk_group_norm_bwd(ctx, q, dy, x, gamma, beta, stats, dx, dg, db)
    sb, sg = total(lambda a, d: d), total(lambda a, d: d * (a - mean) * rstd)
    assert abs(float(db) - sb) <= ULPS * total(lambda a, d: d.abs())
    assert abs(float(dg) - sg) <= ULPS * total(lambda a, d: (d * (a - mean) * rstd).abs())
    for i in range(0, pix, step):
        a, d = x.view(-1)[i:i + step].double(), dy.view(-1)[i:i + step].double()
        xh = (a - mean) * rstd
        assert float((y.view(-1)[i:i + step].double() - (xh * 1.5 + 0.25)).abs().max()) <= 2.0 ** -8 * 12
        want = rstd * 1.5 * (d - sb / pix - xh * sg / pix)
        assert float((dx.view(-1)[i:i + step].double() - want).abs().max()) <= 2.0 ** -8 * 12
    assert dk.dk_device_status(ctx) == 0
