"""The orthogonalised update against the formula in 64 bits.

Tolerances.  Each of the 15 products of five steps is off by at most ~2^-20 of its terms (two fp16 terms per operand,
truncating additions over short chunks); a perturbation of the singular values passes on through the remaining steps
with the polynomial's slope, at most |p'| <= 1.6 where they have settled, and unchanged relative to them while they
grow: 15 * 2^-20 * 1.6^4 ~ 1e-4 in the 2-norm.  A bf16 result adds half a unit of its 8 bits (2^-9, 2^-8 taken)."""
import pytest
import torch

from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
TYPES = {"f32": (dk.DK_F32, torch.float32), "bf16": (dk.DK_BF16, torch.bfloat16)}
QUINTIC, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)
EPS = 1e-7


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    c.close()


def exact(x, steps=5, coefs=QUINTIC, eps=EPS):
    out = []
    for v in x.double():
        w = v if v.shape[0] <= v.shape[1] else v.T
        y = w / (w.norm() + eps)
        for _ in range(steps):
            a = y @ y.T
            y = coefs[0] * y + coefs[1] * (a @ y) + coefs[2] * (a @ (a @ y))
        out.append(y if w is v else y.T)
    return torch.stack(out)


def call(ctx, x, dt, steps=5, coefs=QUINTIC, eps=EPS, scale=1.0, keep=0.0, out=None):
    b, m, n = x.shape
    q = dk.dk_ortho(b, m, n, dt, steps, *coefs, eps)
    ctx.ensure_workspace(q)
    out = torch.full_like(x, float("nan")) if out is None else out
    dk.dk_orthogonalize(ctx, q, x, scale, keep, out)
    return out


def draw(b, m, n, dtype, seed=1, kind="noise"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((b, m, n), generator=g, device="cuda")
    if kind == "decay":         # a few strong directions over a floor of noise, as a gradient has
        r = min(m, n, 8)
        x = 0.05 * x + torch.randn((b, m, r), generator=g, device="cuda") @ torch.randn((b, r, n), generator=g, device="cuda")
    return x.to(dtype)


SHAPES = [(1, 1, 1), (1, 1, 50), (2, 50, 1), (1, 8, 8), (3, 7, 13), (1, 64, 576), (2, 128, 27), (1, 257, 300),
          (1, 300, 257), (4, 100, 1000), (1, 513, 129), (1, 96, 5000), (1, 5000, 96), (2, 640, 640), (1, 1000, 2310)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["noise", "decay"])
@pytest.mark.parametrize("b,m,n", SHAPES)
def test_against_the_formula(ctx, b, m, n, kind, dtype):
    dt, tt = TYPES[dtype]
    x = draw(b, m, n, tt, kind=kind)
    got, want = call(ctx, x, dt), exact(x)
    tol = 2.0 ** -8 if dtype == "bf16" else 1e-4
    for g, w in zip(got, want):
        assert float((g.double() - w).norm()) <= tol * float(w.norm())
    assert dk.dk_device_status(ctx) == 0


# large tiles with and without slices of the contraction; a short side whose columns do not fit in all SMs at once; more
# matrices than SMs; gangs of CTAs of every kind
PATHS = [(1, 2300, 2500), (1, 2500, 2300), (1, 16, 60000), (1, 60000, 16), (200, 8, 300), (30, 64, 640), (1, 128, 18900),
         (1, 128, 33000), (2, 40, 70), (1, 128, 128), (1, 129, 700), (1, 65, 64), (5, 200, 1500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,m,n", PATHS)
def test_every_way_through(ctx, b, m, n, dtype):
    dt, tt = TYPES[dtype]
    x = draw(b, m, n, tt, seed=11, kind="decay")
    got, want = call(ctx, x, dt), exact(x)
    tol = 2.0 ** -8 if dtype == "bf16" else 1e-4
    for g, w in zip(got, want):
        assert float((g.double() - w).norm()) <= tol * float(w.norm())
    assert dk.dk_device_status(ctx) == 0
    assert torch.equal(got, call(ctx, x, dt))


def test_interleaved_with_other_calls(ctx):
    """Calls that use the context's counters and the workspace one after the other, none waited for."""
    x, y = draw(1, 64, 576, torch.float32, seed=12), draw(3, 100, 900, torch.float32, seed=13)
    h = torch.randn((4, 60, 60, 32), device="cuda")
    q = dk.dk_norm(4, 60, 60, 32, 4, 1, 0, 1e-5)
    gamma, beta, stats = torch.ones(32, device="cuda"), torch.zeros(32, device="cuda"), torch.empty((4, 4, 2), device="cuda")
    for p in (q, dk.dk_ortho(3, 100, 900, 0, 5, *QUINTIC, EPS)):
        ctx.ensure_workspace(p)
    want = []
    for i in range(6):
        z = torch.empty_like(h)
        a = call(ctx, x, dk.DK_F32)
        ctx.ensure_workspace(q)
        dk.dk_group_norm_fwd(ctx, q, h, gamma, beta, z, stats)
        b = call(ctx, y, dk.DK_F32)
        want.append((a, z, b))
    for got in want[1:]:
        assert all(torch.equal(u, v) for u, v in zip(got, want[0]))


def test_in_a_graph(ctx):
    """Captured and replayed on other values: nothing but the launches is kept."""
    cases = [draw(1, 64, 576, torch.float32, seed=14), draw(1, 300, 700, torch.float32, seed=15)]
    for x in cases:
        out = call(ctx, x, dk.DK_F32)
        q = dk.dk_ortho(*x.shape, dk.DK_F32, 5, *QUINTIC, EPS)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dk.dk_orthogonalize(ctx, q, x, 1.0, 0.0, out)
        x.copy_(draw(*x.shape, torch.float32, seed=16))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(ctx, x, dk.DK_F32))


def test_singular_values_are_brought_together(ctx):
    """Five steps of the quintic take every singular value of a well-conditioned matrix into [0.65, 1.25]."""
    x = draw(1, 200, 900, torch.float32, seed=2)
    s = torch.linalg.svdvals(call(ctx, x, dk.DK_F32)[0].double())
    assert 0.65 < float(s.min()) and float(s.max()) < 1.25


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 10])
@pytest.mark.parametrize("m,n", [(70, 90), (90, 70)])
def test_steps_and_other_coefficients(ctx, steps, m, n):
    x = draw(2, m, n, torch.float32, seed=3)
    for coefs in (QUINTIC, CUBIC):
        got, want = call(ctx, x, dk.DK_F32, steps, coefs), exact(x, steps, coefs)
        assert float((got.double() - want).norm()) <= 2e-4 * float(want.norm())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps,m,n", [(5, 130, 270), (5, 333, 201), (0, 130, 271), (5, 4, 3000)])
def test_applied_to_weights(ctx, dtype, steps, m, n):
    """out = keep*out + scale*X with `out` the weights."""
    dt, tt = TYPES[dtype]
    x, w = draw(2, m, n, tt, seed=4), draw(2, m, n, tt, seed=5)
    got = call(ctx, x, dt, steps, scale=-0.3, keep=0.99, out=w.clone())
    want = 0.99 * w.double() - 0.3 * exact(x, steps)
    tol = 2.0 ** -8 if dtype == "bf16" else 1e-4
    assert float((got.double() - want).norm()) <= tol * float(want.norm())
    # keep = 0 does not read `out`
    got = call(ctx, x, dt, steps, scale=2.0, out=torch.full_like(w, float("nan")))
    assert bool(torch.isfinite(got).all())


@pytest.mark.parametrize("magnitude", [1e-30, 1e-12, 1e15])
def test_any_magnitude(ctx, magnitude):
    x = draw(1, 90, 200, torch.float32, seed=6)
    got, want = call(ctx, x * magnitude, dk.DK_F32, eps=0.0), exact(x * magnitude, eps=0.0)
    assert float((got.double() - want).norm()) <= 1e-4 * float(want.norm())


def test_zero_and_rank_one(ctx):
    x = torch.zeros((3, 40, 60), device="cuda")
    x[1] = torch.outer(torch.linspace(-1, 1, 40, device="cuda"), torch.linspace(1, 2, 60, device="cuda"))
    x[2, 3, 7] = -5.0
    got, want = call(ctx, x, dk.DK_F32), exact(x)
    assert float(got[0].abs().max()) == 0.0
    for i in (1, 2):
        assert float((got[i].double() - want[i]).norm()) <= 1e-4 * float(want[i].norm())


def test_non_finite_values_stay_in_their_matrix(ctx):
    x = draw(3, 64, 100, torch.float32, seed=7)
    clean = call(ctx, x, dk.DK_F32)
    x[1, 5, 6] = float("nan")
    got = call(ctx, x, dk.DK_F32)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])
    assert bool(torch.isnan(got[1]).all())


def test_repeats_bit_for_bit(ctx):
    for shape in ((1, 64, 576), (2, 300, 700), (1, 700, 300)):
        x = draw(*shape, torch.float32, seed=8)
        assert torch.equal(call(ctx, x, dk.DK_F32), call(ctx, x, dk.DK_F32))


def test_another_stream(ctx):
    x = draw(1, 128, 1152, torch.float32, seed=9)
    want = call(ctx, x, dk.DK_F32)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call(ctx, x, dk.DK_F32)
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals(ctx):
    x = draw(1, 8, 8, torch.float32)
    q = dk.dk_ortho(1, 8, 8, dk.DK_F32, 5, *QUINTIC, EPS)
    ctx.ensure_workspace(q)
    with pytest.raises(dk.DkError) as e:
        dk.dk_orthogonalize(ctx, q, x, 1.0, 0.0, x)
    assert e.value.status == 1
    with pytest.raises(ValueError):
        dk.dk_orthogonalize(ctx, q, x.double(), 1.0, 0.0, torch.empty_like(x))
    with pytest.raises(ValueError):
        dk.dk_orthogonalize(ctx, q, x, 1.0, 0.0, torch.empty((1, 8, 9), device="cuda"))
    fresh = dk.Context(0)
    with pytest.raises(dk.DkError) as e:
        dk.dk_orthogonalize(fresh, q, x, 1.0, 0.0, torch.empty_like(x))
    assert e.value.status == 4
    fresh.close()


def test_expired_wait_is_reported(ctx):
    x = draw(1, 300, 700, torch.float32, seed=10)
    dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 12)
    dk.dk_set_option(ctx, dk.DK_OPT_TEST_WITHHOLD, 1)
    try:
        call(ctx, x, dk.DK_F32)
        assert dk.dk_device_status(ctx) == dk.DK_ERR_TIMEOUT
    finally:
        dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 22)
    got, want = call(ctx, x, dk.DK_F32), exact(x)
    assert float((got.double() - want).norm()) <= 1e-4 * float(want.norm())


@pytest.mark.parametrize("b,m,n,steps", [(1, 64, 576, 12), (1, 48, 1100, 12), (3, 576, 64, 8), (1, 100, 250, 12),
                                         (1, 30, 3900, 9), (2, 90, 2000, 8)])
def test_gangs_beside_other_work(ctx, b, m, n, steps):
    """Gangs that add their shares up directly meet once a step (the last case: twice).  What delays single CTAs of a
    gang, traffic and kernels of another stream, must not mix the shares of two steps: every result has the same bits."""
    x = draw(b, m, n, torch.float32, seed=17)
    want = call(ctx, x, dk.DK_F32, steps, CUBIC)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big, small = torch.empty(1 << 27, device="cuda"), torch.randn((300, 300), device="cuda")
    outs = []
    for i in range(40):
        with torch.cuda.stream(side):
            big.mul_(1.0)
            for _ in range(4):
                small @ small
        outs.extend(call(ctx, x, dk.DK_F32, steps, CUBIC) for _ in range(10))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    assert dk.dk_device_status(ctx) == 0


@pytest.mark.parametrize("m,n", [(90, 200), (200, 90), (300, 700), (300, 701)])
def test_ends_of_the_range(ctx, m, n):
    """Matrices whose norm is near either end of fp32's range (the small ones from numbers of few bits, so that being
    subnormal costs them none), and a zero matrix with an eps as small."""
    x = draw(1, m, n, torch.bfloat16, seed=18).float()
    x = torch.where(x.abs() < 2.0 ** -5, torch.zeros_like(x), x)
    small, large = (x * 2.0 ** -70 * 2.0 ** -64).contiguous(), (x * 2.0 ** 124).contiguous()
    assert torch.equal(small.double(), x.double() * 2.0 ** -134)
    for v in (small, large):
        got, want = call(ctx, v, dk.DK_F32, eps=0.0), exact(v, eps=0.0)
        assert float((got.double() - want).norm()) <= 1e-4 * float(want.norm())
    x[:] = 0
    assert float(call(ctx, x, dk.DK_F32, eps=1e-38).abs().max()) == 0.0
    x[0, 3, 5] = 2.0 ** -120
    got, want = call(ctx, x, dk.DK_F32, eps=1e-38), exact(x, eps=1e-38)
    assert float((got.double() - want).norm()) <= 1e-4 * float(want.norm())
