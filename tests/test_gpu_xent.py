"""Linear layer with softmax cross entropy against the formula in 64 bits.

Tolerances.  A logit is a sum of d products.  fp32 operands enter as two fp16 terms: each is off by at most 2^-22 of
itself, the dropped product of the low terms by 2^-22, and the tensor pipe's truncating additions by 24 units of 2^-24
per chunk: below 2^-19 of sum |h||W| together.  bf16 operands are exact, only the additions count (64 per chunk): the
same bound holds.  lse and loss are off by twice that and a few fp32 roundings of their own size.  A probability is
off by the same amount relative to itself; the gradients add the roundings of p (2^-9 of each term with bf16, 2^-21
with fp32), their own products, and the rounding of the result (2^-9 with bf16).  The gradients are compared in the
2-norm."""
import pytest
import torch

from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
TYPES = {"f32": (dk.DK_F32, torch.float32), "bf16": (dk.DK_BF16, torch.bfloat16)}


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    c.close()


def draw(rows, d, vocab, dtype, seed=1, gain=2.0, ignored=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((rows, d), generator=g, device="cuda")
    W = torch.randn((vocab, d), generator=g, device="cuda") * (gain / d ** 0.5)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    t = torch.where(torch.rand(rows, generator=g, device="cuda") < ignored, torch.full_like(t, -1), t)
    return h.to(dtype), W.to(dtype), t


def exact(h, W, t, dloss=None, scale=1.0):
    h, W = h.double(), W.double()
    keep = (t >= 0) & (t < W.shape[0])
    h = torch.where(keep[:, None], h, torch.zeros_like(h))
    z = h @ W.T
    lse = torch.logsumexp(z, dim=1)
    at = torch.where(keep, t, torch.zeros_like(t))[:, None]
    loss = lse - z.gather(1, at)[:, 0]
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, at, torch.full(at.shape, -1.0, dtype=p.dtype, device=p.device))
    g = torch.full_like(lse, scale) if dloss is None else scale * dloss.double()
    p = p * torch.where(keep, g, torch.zeros_like(g))[:, None]
    zero = torch.zeros_like(lse)
    return torch.where(keep, loss, zero), torch.where(keep, lse, zero), p @ W, p.T @ h


def call(ctx, h, W, t, dt, dloss=None, scale=1.0, lse_in=None):
    q = dk.dk_xent(h.shape[0], h.shape[1], W.shape[0], dt)
    ctx.ensure_workspace(q)
    nan = float("nan")
    loss = torch.full((h.shape[0],), nan, device="cuda")
    lse = torch.full((h.shape[0],), nan, device="cuda")
    dh, dW = torch.full_like(h, nan), torch.full_like(W, nan)
    dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
    dk.dk_linear_xent_bwd(ctx, q, h, W, t, lse, dloss, scale, dh, dW)
    return loss, lse, dh, dW


def check(ctx, h, W, t, dtype, dloss=None, scale=1.0):
    dt = TYPES[dtype][0]
    loss, lse, dh, dW = call(ctx, h, W, t, dt, dloss, scale)
    want = exact(h, W, t, dloss, scale)
    keep = (t >= 0) & (t < W.shape[0])
    hz = torch.where(keep[:, None], h.double(), torch.zeros_like(h.double()))
    tol = 2.0 ** -19 * float((hz.abs() @ W.double().abs().T).max())
    bound = 2 * tol + 8 * 2.0 ** -24 * (1 + want[1].abs())
    assert bool(((lse.double() - want[1]).abs() <= bound).all())
    assert bool(((loss.double() - want[0]).abs() <= bound + 8 * 2.0 ** -24 * want[0].abs()).all())
    # p = softmax - onehot is formed by a subtraction whose error is relative to one: it counts where p itself is small
    rel = 2 * tol + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -18)
    g = float((torch.ones_like(lse) if dloss is None else dloss).abs().max()) * abs(scale)
    floor = 2.0 ** -22 * g
    assert float((dh.double() - want[2]).norm()) <= rel * float(want[2].norm()) + floor * float(W.double().norm())
    assert float((dW.double() - want[3]).norm()) <= rel * float(want[3].norm()) + floor * float(hz.norm())
    assert dk.dk_device_status(ctx) == 0
    return loss, lse, dh, dW


SHAPES = [(1, 1, 1), (1, 16, 10), (3, 7, 2), (64, 512, 1000), (5, 100, 257), (130, 64, 255), (257, 13, 300),
          (300, 1000, 129), (1, 4096, 513), (1000, 8, 10), (33, 65, 5001), (2047, 72, 641), (512, 520, 7000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,vocab", SHAPES)
def test_against_the_formula(ctx, rows, d, vocab, dtype):
    h, W, t = draw(rows, d, vocab, TYPES[dtype][1])
    if rows < 4:
        t.clamp_(min=0)
    check(ctx, h, W, t, dtype, scale=1.0 / rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_row_weights(ctx, dtype):
    h, W, t = draw(200, 96, 700, TYPES[dtype][1], seed=2)
    g = torch.Generator(device="cuda").manual_seed(3)
    dloss = torch.randn(200, generator=g, device="cuda")
    dloss[5] = 0.0
    _, _, dh, _ = check(ctx, h, W, t, dtype, dloss=dloss, scale=-0.25)
    assert float(dh[5].abs().max()) == 0.0
    # nothing asked for: zero gradients, no NaN from a largest magnitude of zero
    _, _, dh, dW = call(ctx, h, W, t, TYPES[dtype][0], dloss=torch.zeros_like(dloss))
    assert float(dh.abs().max()) == 0.0 and float(dW.abs().max()) == 0.0


@pytest.mark.parametrize("dtype,rows,d,vocab", [("f32", 2048, 40, 40000), ("bf16", 4096, 24, 33001)])
def test_several_pieces_of_the_vocabulary(ctx, dtype, rows, d, vocab):
    h, W, t = draw(rows, d, vocab, TYPES[dtype][1], seed=4)
    check(ctx, h, W, t, dtype, scale=1.0 / rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [70, 600])
def test_rows_left_out_are_not_read(ctx, dtype, rows):
    """NaN, infinities and the type's extremes in rows that are left out reach neither the losses, nor dh, nor dW."""
    h, W, t = draw(rows, 48, 900, TYPES[dtype][1], seed=5, ignored=0.5)
    t[0], t[1], t[2], t[3] = -1, -100, -2 ** 62, 4
    clean = call(ctx, h, W, t, TYPES[dtype][0])
    out = (t < 0).nonzero()[:, 0]
    for i, bad in enumerate((float("nan"), float("inf"), -float("inf"), torch.finfo(h.dtype).max)):
        h[out[i::4]] = bad
    got = call(ctx, h, W, t, TYPES[dtype][0])
    for a, b in zip(got, clean):
        assert torch.equal(a, b)
    assert float(got[0][out].abs().max()) == 0 and float(got[1][out].abs().max()) == 0
    assert float(got[2][out].abs().max()) == 0
    assert all(bool(torch.isfinite(a).all()) for a in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_row_left_out(ctx, dtype):
    h, W, t = draw(40, 32, 100, TYPES[dtype][1], seed=6)
    h[:] = float("nan")
    got = call(ctx, h, W, torch.full_like(t, -1), TYPES[dtype][0])
    assert all(float(a.abs().max()) == 0 for a in got)


@pytest.mark.parametrize("rows", [20, 700])
def test_target_past_the_vocabulary_is_reported(ctx, rows):
    h, W, t = draw(rows, 32, 600, torch.float32, seed=7, ignored=0.0)
    t[3], t[7] = 600, 2 ** 40
    got = call(ctx, h, W, t, dk.DK_F32)
    assert dk.dk_device_status(ctx) == 1                        # DK_ERR_INVALID_ARG
    assert dk.dk_device_status(ctx) == 0                        # read and cleared
    want = exact(h, W, t)
    assert float(got[0][3]) == 0 and float(got[0][7]) == 0 and float(got[2][3].abs().max()) == 0
    assert float((got[3].double() - want[3]).norm()) <= 1e-5 * float(want[3].norm())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gain", [1e-6, 200.0, 3000.0])
def test_logits_of_any_size(ctx, dtype, gain):
    """Tiny logits (a flat softmax) and huge ones (exp of the raw logit would overflow)."""
    h, W, t = draw(300, 64, 800, TYPES[dtype][1], seed=8, gain=gain)
    loss, lse, _, _ = call(ctx, h, W, t, TYPES[dtype][0])
    want = exact(h, W, t)
    tol = 2.0 ** -18 * float((h.double().abs() @ W.double().abs().T).max()) + 1e-6
    assert bool(((lse.double() - want[1]).abs() <= tol * (1 + 1e-7 * want[1].abs())).all())
    assert bool(((loss.double() - want[0]).abs() <= 2 * tol).all())


@pytest.mark.parametrize("scale_h,scale_w", [(1e-15, 1e10), (1e12, 1e-20), (1e-30, 1.0)])
def test_operands_of_any_magnitude(ctx, scale_h, scale_w):
    """The common power of two of an fp32 operand follows its largest magnitude."""
    h, W, t = draw(300, 64, 500, torch.float32, seed=9)
    h, W = h * scale_h, W * scale_w
    loss, lse, dh, dW = call(ctx, h, W, t, dk.DK_F32)
    want = exact(h, W, t)
    tol = 2.0 ** -18 * float((h.double().abs() @ W.double().abs().T).max()) + 2e-6
    assert float((lse.double() - want[1]).abs().max()) <= tol * 2
    assert float((dh.double() - want[2]).norm()) <= (2.0 ** -17 + 4 * tol) * float(want[2].norm())
    assert float((dW.double() - want[3]).norm()) <= (2.0 ** -17 + 4 * tol) * float(want[3].norm())


def test_magnitudes_that_differ_within_a_tensor(ctx):
    """Features whose scales differ by 2^16 keep their bits: the terms hold 22 of them down to 2^-18 of the largest."""
    h, W, t = draw(260, 64, 520, torch.float32, seed=10)
    s = 2.0 ** torch.linspace(0, 16, 64, device="cuda").round()
    check(ctx, (h * s).contiguous(), (W / s).contiguous(), t, "f32")


def test_gradient_against_differences(ctx):
    """<dh, u> and <dW, v> against central differences of the weighted loss in 64 bits (step 1e-4: off by ~1e-8)."""
    h, W, t = draw(40, 24, 90, torch.float32, seed=11)
    g = torch.Generator(device="cuda").manual_seed(12)
    dloss = torch.rand(40, generator=g, device="cuda")
    _, _, dh, dW = call(ctx, h, W, t, dk.DK_F32, dloss=dloss, scale=0.5)
    u = torch.randn(h.shape, generator=g, device="cuda", dtype=torch.float64)
    v = torch.randn(W.shape, generator=g, device="cuda", dtype=torch.float64)
    step = 1e-4

    def f(a, b):
        return float((exact(h.double() + a * u, W.double() + b * v, t)[0] * dloss.double()).sum() * 0.5)

    for grad, dirn, diff in ((dh, u, (f(step, 0) - f(-step, 0)) / (2 * step)),
                             (dW, v, (f(0, step) - f(0, -step)) / (2 * step))):
        terms = (grad.double() * dirn)
        assert abs(float(terms.sum()) - diff) <= 2e-5 * float(terms.abs().sum())


def test_repeats_bit_for_bit(ctx):
    for shape in ((64, 512, 1000), (600, 200, 3000)):
        h, W, t = draw(*shape, torch.float32, seed=13)
        a, b = call(ctx, h, W, t, dk.DK_F32), call(ctx, h, W, t, dk.DK_F32)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_no_rows(ctx):
    q = dk.dk_xent(0, 16, 30, dk.DK_F32)
    ctx.ensure_workspace(q)
    e, t, f = torch.empty((0, 16), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    W, dW = torch.ones((30, 16), device="cuda"), torch.ones((30, 16), device="cuda")
    dk.dk_linear_xent_fwd(ctx, q, e, W, t, f, f)
    dk.dk_linear_xent_bwd(ctx, q, e, W, t, f, None, 1.0, e, dW)
    assert float(dW.abs().max()) == 0


def test_offsets_past_32_bits(ctx):
    """W and dW of more than 2^31 bytes and vocab*d past 2^30 elements: the last classes are checked by themselves."""
    rows, d, vocab = 64, 4096, 530000
    g = torch.Generator(device="cuda").manual_seed(14)
    h = torch.randn((rows, d), generator=g, device="cuda", dtype=torch.bfloat16)
    W = torch.randn((vocab, d), generator=g, device="cuda", dtype=torch.bfloat16)
    W.mul_(2.0 / d ** 0.5)
    assert vocab * d > 2 ** 31
    t = torch.full((rows,), vocab - 1, dtype=torch.int64, device="cuda") - torch.arange(rows, device="cuda")
    loss, lse, dh, dW = call(ctx, h, W, t, dk.DK_BF16)
    z = torch.cat([h.double() @ W[i:i + 53000].double().T for i in range(0, vocab, 53000)], dim=1)
    want = torch.logsumexp(z, dim=1)
    assert float((lse.double() - want).abs().max()) <= 2.0 ** -18 * 4 * d ** 0.5
    p = torch.exp(z[:, -rows:] - want[:, None])
    p[torch.arange(rows), t - (vocab - rows)] -= 1
    last = p.T @ h.double()
    assert float((dW[-rows:].double() - last).norm()) <= 2.0 ** -7 * float(last.norm())
    assert bool(torch.isfinite(dh).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d,vocab", [(50, 64, 900), (900, 256, 4000)])
def test_in_a_graph(ctx, dtype, rows, d, vocab):
    """Captured and replayed on other values: nothing but the launches is kept."""
    dt, tt = TYPES[dtype]
    h, W, t = draw(rows, d, vocab, tt, seed=17)
    loss, lse, dh, dW = call(ctx, h, W, t, dt)
    q = dk.dk_xent(rows, d, vocab, dt)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
        dk.dk_linear_xent_bwd(ctx, q, h, W, t, lse, None, 1.0, dh, dW)
    h2, W2, t2 = draw(rows, d, vocab, tt, seed=18)
    h.copy_(h2); W.copy_(W2); t.copy_(t2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((loss, lse, dh, dW), call(ctx, h, W, t, dt)))


def test_many_rows(ctx):
    """So many rows that a piece is a few hundred classes wide."""
    h, W, t = draw(150000, 16, 1400, torch.float32, seed=19)
    check(ctx, h, W, t, "f32", scale=1e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8, 9])
@pytest.mark.parametrize("d,vocab", [(1, 1), (64, 33), (255, 1000), (258, 4097), (512, 20011), (1024, 60000), (4096, 700),
                                     (2047, 300), (12288, 90), (30000, 40)])
def test_few_rows(ctx, rows, d, vocab, dtype):
    """A token or a handful, at lengths around a warp's step and vocabularies with and without classes for every warp."""
    h, W, t = draw(rows, d, vocab, TYPES[dtype][1], seed=20, ignored=0.3)
    t[-1] = vocab - 1
    check(ctx, h, W, t, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_rows_extremes(ctx, dtype):
    """A row that is left out keeps its NaN to itself, another's infinity or lowest value does what the formula says."""
    dt, tt = TYPES[dtype]
    h, W, _ = draw(6, 128, 3000, tt, seed=21)
    t = torch.tensor([5, -1, 2999, 0, 3000, 7], device="cuda")
    h[1], h[4, 3] = float("nan"), float("inf")
    h[3] = 0
    W[11] = 0
    W[11, 0] = torch.finfo(tt).min / 2          # the class's logit is far below all others, or far above
    h[0, 0], h[2, 0], h[5, 0] = 1.0, 1.0, 1.0
    q = dk.dk_xent(6, 128, 3000, dt)
    ctx.ensure_workspace(q)
    loss, lse = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
    want = exact(h, W, t)
    for r in (0, 2, 3, 5):
        assert abs(float(lse[r].double() - want[1][r])) <= 1e-4 and abs(float(loss[r].double() - want[0][r])) <= 1e-4
    for r in (1, 4):
        assert float(loss[r]) == 0 and float(lse[r]) == 0
    assert dk.dk_device_status(ctx) == 1                        # DK_ERR_INVALID_ARG
    h[5, 0] = float("nan")
    dk.dk_linear_xent_fwd(ctx, q, h, W, torch.tensor([5, -1, 2999, 0, -1, 7], device="cuda"), loss, lse)
    assert bool(torch.isnan(loss[5])) and bool(torch.isnan(lse[5])) and not bool(torch.isnan(loss[:5]).any())
    assert dk.dk_device_status(ctx) == 0


def test_another_stream(ctx):
    h, W, t = draw(300, 128, 2000, torch.bfloat16, seed=15)
    want = call(ctx, h, W, t, dk.DK_BF16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call(ctx, h, W, t, dk.DK_BF16)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(ctx):
    h, W, t = draw(8, 16, 30, torch.float32)
    f = torch.empty(8, device="cuda")
    q = dk.dk_xent(8, 16, 30, dk.DK_F32)
    ctx.ensure_workspace(q)
    with pytest.raises(ValueError):
        dk.dk_linear_xent_fwd(ctx, q, h, W, t.to(torch.int32), f, f.clone())
    with pytest.raises(ValueError):
        dk.dk_linear_xent_fwd(ctx, q, h.to(torch.bfloat16), W, t, f, f.clone())
    with pytest.raises(ValueError):
        dk.dk_linear_xent_fwd(ctx, q, h[:4], W, t, f, f.clone())
    with pytest.raises(ValueError):
        dk.dk_linear_xent_fwd(ctx, q, h.t(), W, t, f, f.clone())
    fresh = dk.Context(0)
    with pytest.raises(dk.DkError) as e:
        dk.dk_linear_xent_fwd(fresh, q, h, W, t, f, f.clone())
    assert e.value.status == 4                                  # DK_ERR_WORKSPACE
    fresh.close()


@pytest.mark.parametrize("rows,d,vocab", [(300, 256, 2000), (16, 4096, 100)])
def test_expired_wait_is_reported(ctx, rows, d, vocab):
    """The producer of one product arms a stage and copies nothing: every wait runs out, the status says so, the
    next call is correct (both the product with its epilogue and the sliced one)."""
    h, W, t = draw(rows, d, vocab, torch.float32, seed=16)
    dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 12)
    dk.dk_set_option(ctx, dk.DK_OPT_TEST_WITHHOLD, 1)
    try:
        call(ctx, h, W, t, dk.DK_F32)
        assert dk.dk_device_status(ctx) == dk.DK_ERR_TIMEOUT
    finally:
        dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 22)
    check(ctx, h, W, t, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("magnitude", [1.0, 1e5, 1e-5])
@pytest.mark.parametrize("rows,vocab", [(20, 500), (300, 500), (2000, 6000)])
def test_non_finite_values_stay_in_their_row(ctx, rows, vocab, magnitude, dtype):
    """A row that takes part and holds a NaN or an infinity, or whose weight is one: its loss and dh are NaN, and dW, to
    which it belongs; every other row has the bits that it has without it, whatever the operands' magnitudes."""
    dt, tt = TYPES[dtype]
    h, W, t = draw(rows, 64, vocab, torch.float32, seed=23, ignored=0.1)
    t[7] = 3
    h[7, 5] = 0.0                                              # (not the largest magnitude)
    dloss = torch.ones(rows, device="cuda")
    dloss[8] = 2.0
    h, W = (h * magnitude).to(tt), (W / magnitude).to(tt)
    others = torch.arange(rows, device="cuda") != 7
    clean = call(ctx, h, W, t, dt, dloss=dloss)
    for bad in (float("nan"), float("inf"), -float("inf")):
        h2, d2 = h.clone(), dloss.clone()
        h2[7, 5], d2[7] = bad, bad
        for got, own in ((call(ctx, h2, W, t, dt, dloss=dloss), (0, 1, 2)), (call(ctx, h, W, t, dt, dloss=d2), (2,))):
            for i in range(3):
                assert torch.equal(got[i][others], clean[i][others])
                assert not bool(torch.isfinite(got[i][7]).any()) if i in own else torch.equal(got[i][7], clean[i][7])
            assert not bool(torch.isfinite(got[3]).any())
    assert dk.dk_device_status(ctx) == 0


@pytest.mark.parametrize("rows,d,vocab", [(9, 64, 600), (200, 64, 600), (64, 512, 1000), (3000, 300, 4001), (9, 30000, 200),
                                          (2100, 40, 40000), (300, 2000, 2600)])
@pytest.mark.parametrize("scale_h,scale_w,weight", [(1.0, 1.0, 1.0), (2.0 ** -80, 2.0 ** 80, 2.0 ** -30),
                                                    (2.0 ** 70, 2.0 ** -70, 2.0 ** 40)])
def test_improbable_classes_keep_their_digits(ctx, rows, d, vocab, scale_h, scale_w, weight):
    """dW row by row, for classes whose probability falls to 1e-17 in every row: each row's error is relative to its own
    terms.  A probability is off by twice the logits' error (2^-19 of the terms, as above) and exp's own rounding
    (2^-22 of its argument); the two terms add 2^-22 of the class's largest probability per row, h and the sums 2^-19."""
    h, W, t = draw(rows, d, vocab, torch.float32, seed=24, gain=0.5)
    g = torch.Generator(device="cuda").manual_seed(25)
    h[:, 0] = 1.0
    W[:, 0] = -40.0 * torch.rand(vocab, generator=g, device="cuda")
    W[:8, 0] = 0.0
    t = torch.where(t >= 0, t % 8, t)                          # targets among the probable classes
    h, W = h * scale_h, W * scale_w
    dloss = weight * (0.5 + torch.rand(rows, generator=g, device="cuda"))
    loss, lse, dh, dW = call(ctx, h, W, t, dk.DK_F32, dloss=dloss)
    want = exact(h, W, t, dloss=dloss)
    keep = t >= 0
    hk, tk = h.double()[keep], t[keep]
    z = hk @ W.double().T
    p = torch.exp(z - torch.logsumexp(z, dim=1)[:, None])
    assert float(p.max(dim=0).values.min()) < 1e-15
    p[torch.arange(len(tk), device="cuda"), tk] = 1.0          # (1 - p there: relative to one)
    p *= dloss.double()[keep][:, None]
    size = hk.norm(dim=1)
    rel = 2.0 ** -18 * float((hk.abs() @ W.double().abs().T).max()) + 2.0 ** -22 * 60 + 2.0 ** -18
    bound = rel * (p.T @ size) + 2.0 ** -22 * p.max(dim=0).values * size.sum()
    bound += 2.0 ** -149 * d ** 0.5                            # (where the result itself is subnormal)
    err = (dW.double() - want[3]).norm(dim=1)
    assert bool((err <= bound).all())
    assert float((dh.double() - want[2]).norm()) <= rel * float(want[2].norm()) + 2.0 ** -22 * weight * float(W.double().norm())


@pytest.mark.parametrize("dtype,rows,d,few", [
    ("f32", 1, 8192, True), ("f32", 1, 8193, False), ("f32", 1, 8160, True), ("f32", 2, 6144, True), ("f32", 4, 6143, True),
    ("f32", 4, 6112, True), ("f32", 4, 6145, False), ("f32", 3, 6160, False), ("f32", 5, 3071, True), ("f32", 8, 3040, True),
    ("f32", 8, 3071, True), ("f32", 8, 3073, False), ("f32", 5, 3088, False), ("f32", 9, 64, False),
    ("bf16", 1, 8192, True), ("bf16", 1, 8191, True), ("bf16", 1, 8200, False), ("bf16", 2, 64, False)])
def test_limits_of_the_dot_products(ctx, dtype, rows, d, few):
    """Either side of each limit that dk.h states, and which way was taken: the dot products are two kernels (with the one
    that joins), the tensor cores' way one more where operands are laid out (fp32, or rows off 16-byte boundaries)."""
    h, W, t = draw(rows, d, 300, TYPES[dtype][1], seed=26, ignored=0.0)
    check(ctx, h, W, t, dtype)
    q = dk.dk_xent(rows, d, 300, TYPES[dtype][0])
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dk.dk_profile_reset(ctx)
    dk.dk_linear_xent_fwd(ctx, q, h, W, t, loss, lse)
    launches = dk.dk_profile_read(ctx)["other"][2]
    assert launches == (2 if few or (dtype == "bf16" and d % 8 == 0) else 3)


@pytest.mark.parametrize("dtype,rows", [("f32", 1), ("f32", 3), ("f32", 8), ("bf16", 1)])
@pytest.mark.parametrize("margin", [5.0, 10.0, 15.0, 20.0])
@pytest.mark.parametrize("d,vocab", [(256, 1000), (255, 3001), (1024, 30000)])
def test_sure_rows(ctx, dtype, rows, margin, d, vocab):
    """Rows whose target's probability is almost one: what is left of p there is a difference.  Both directions form a
    row's logits alike, so what p misses at the target is lse's rounding and exp's (2^-22), never the logits' own error."""
    tt = TYPES[dtype][1]
    g = torch.Generator(device="cuda").manual_seed(27)
    W = torch.randn((vocab, d), generator=g, device="cuda") / d ** 0.5
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    h = 0.5 * torch.randn((rows, d), generator=g, device="cuda") + W[t] / W[t].norm(dim=1, keepdim=True) ** 2 * (margin + 6)
    h, W = h.to(tt), W.to(tt)
    _, lse, dh, _ = call(ctx, h, W, t, TYPES[dtype][0])
    z = h.double() @ W.double().T
    p = torch.exp(z - torch.logsumexp(z, dim=1)[:, None])
    at = torch.arange(rows, device="cuda")
    p[at, t] = 0
    p[at, t] = -p.sum(dim=1)                                   # (exactly, where 1 - p would cancel)
    want = p @ W.double()
    off = 2.0 ** -22 + 2.0 ** -24 * lse.double().abs()
    rel = 2.0 ** -18 * float((h.double().abs() @ W.double().abs().T).max()) + (2.0 ** -7 if dtype == "bf16" else 2.0 ** -17)
    bound = 2 * off * W.double()[t].norm(dim=1) + rel * (p.abs() @ W.double().abs()).norm(dim=1)
    assert bool(((dh.double() - want).norm(dim=1) <= bound).all())


@pytest.mark.parametrize("scale", [1.0 / 15, 1.0 / 2047, 0.3])
@pytest.mark.parametrize("rows,d,vocab", [(1, 2048, 5000), (100, 64, 5000), (2000, 500, 3000), (3000, 64, 40000), (9, 60000, 400)])
def test_p_is_rounded_without_its_scale(ctx, rows, d, vocab, scale):
    """bf16, a flat softmax: p is nearly -scale at every target, and rounded with the scale in it would take up to 2^-8 off
    the whole gradient.  Element by element: scale times the products of p rounded without it, off by the result's rounding
    (2^-8 of it), by a probability that rounds the other way (2^-8 of the terms that are not targets, whose 1 - 1/vocab is
    not halfway between two bf16 numbers), and by the sums (2^-19 of all terms)."""
    h, W, t = draw(rows, d, vocab, torch.bfloat16, seed=28, gain=0.01, ignored=0.0)
    _, _, dh, dW = call(ctx, h, W, t, dk.DK_BF16, scale=scale)
    hd, Wd, at = h.double(), W.double(), torch.arange(rows, device="cuda")
    z = hd @ Wd.T
    p = torch.exp(z - torch.logsumexp(z, dim=1)[:, None])
    p[at, t] -= 1
    p = p.float().to(torch.bfloat16).double()
    small = p.abs()
    small[at, t] = 0
    live = t.unique()
    for got, want, rest, terms in (
            (dh, p @ Wd, small @ Wd.abs(), p.abs() @ Wd.abs()),
            (dW[live], p[:, live].T @ hd, small[:, live].T @ hd.abs(), p[:, live].abs().T @ hd.abs())):
        bound = scale * (2.0 ** -8 * (want.abs() + 2 * rest) + 2.0 ** -19 * terms)
        assert bool(((got.double() - scale * want).abs() <= bound).all())
