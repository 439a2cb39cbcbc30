"""Checkpoints and the weight gradient from one where they can go wrong at the edges: tiles that end anywhere, columns of very
many rows, infinities, the ends of the 8-bit form's range."""
import pytest
import torch

import kept
from paper_2207_00083_b200 import binding as dk
from test_gpu_ckpt8 import draw, stored, wgrad_bound

pytestmark = pytest.mark.gpu
TYPES = {"f32": (dk.DK_F32, torch.float32), "bf16": (dk.DK_BF16, torch.bfloat16)}


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    assert dk.dk_device_status(c) == 0
    c.close()


# Tiles of 256 x 256 stored by TMA, more of them than CTA pairs (so a warp has several), of few stages each (so stores queue
# up), with 1 to 32 or 65 to 96 columns left of a warp's 128 at the right edge: one or three pieces of 32, by the side of
# tiles that have none left, two or four.
EDGES = [(256, 4128, 4096), (64, 4176, 5000), (256, 1056, 8192), (256, 4192, 11008), (2048, 96, 66000), (64, 2084, 9000),
         (100, 1124, 8192), (1000, 8352, 2304)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", EDGES)
def test_wgrad_tiles_at_the_edge(ctx, rows, d, out, dtype):
    """Every value, and the same bits in every one of many calls without a pause between them: no tile takes the place of
    another on its way out."""
    code, dt = TYPES[dtype]
    x, dy = stored(ctx, draw(rows, d, dt, spread=0.5)), draw(rows, out, dt, seed=5, spread=0.5)
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    results = [torch.full((out, d), float("nan"), device="cuda") for _ in range(6)]
    for dW in results:
        dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, dW, None)
    xv, dyv = kept.decode(x, rows, d), dy.double()
    err = (results[0].double() - dyv.t() @ xv).abs_()
    assert bool((err <= wgrad_bound(dyv, xv, dtype)).all())
    for dW in results[1:]:
        assert torch.equal(dW, results[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,out,parts", [(20000, 38400, 1), (5000000, 16, 153)])
def test_columns_of_many_rows(ctx, rows, out, parts, dtype):
    """db of a wide layer, whose columns are summed in one part of the rows, and of more rows than the usual parts take: a large
    value before many small ones.  A thread has every eighth of a part's rows and sums 64 at a time, then those sums; then
    come eight warps, the parts by eight groups of threads at most and those: so many roundings of 2^-24, and scale's."""
    code, dt = TYPES[dtype]
    d = 32
    x, dy = stored(ctx, draw(rows, d, dt, spread=0.5)), torch.ones((rows, out), dtype=dt, device="cuda")
    dy[0], dy[5, ::2] = 2.0 ** 25, -(2.0 ** 25)
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW, db = torch.empty((out, d), device="cuda"), torch.full((out,), float("nan"), device="cuda")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 0.75, 0.0, dW, db)
    depth = 64 + -(-rows // parts) / 8 / 64 + 8 + parts / 4 + 8
    want, size = (f(dy).sum(dim=0, dtype=torch.float64) * 0.75 for f in (lambda t: t, torch.abs))
    assert bool(((db.double() - want).abs() <= size * (depth + 2) * 2.0 ** -24).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", [(100, 96, 40), (100, 96, 41), (256, 1056, 8192), (33000, 40, 24)])
def test_wgrad_infinities_as_in_the_formula(ctx, rows, d, out, dtype):
    """An infinity in dy times x: infinities of the products' signs, NaN where x is zero or two of them meet; so in db."""
    code, dt = TYPES[dtype]
    dy, x = draw(rows, out, dt, spread=0.5), draw(rows, d, dt, seed=2, spread=0.5)
    inf = float("inf")
    dy[7, 3], dy[9, 11], dy[20, 5], dy[60, 5], dy[2, 6], dy[3, 6], x[7, 8] = inf, -inf, inf, inf, inf, -inf, 0.0
    ckpt = stored(ctx, x)
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW, db = torch.empty((out, d), device="cuda"), torch.empty(out, device="cuda")
    for scale in (1.0, -0.5):
        dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, ckpt, scale, 0.0, dW, db)
        want, want_b = scale * (dy.double().t() @ kept.decode(ckpt, rows, d)), scale * dy.double().sum(dim=0)
        for got, w in ((dW, want), (db, want_b)):
            bad = ~torch.isfinite(w)
            assert torch.equal(~torch.isfinite(got), bad)
            assert torch.equal(got[bad].double().nan_to_num(nan=7.0), w[bad].nan_to_num(nan=7.0))


@pytest.mark.parametrize("dtype", TYPES)
def test_how_far_a_kept_value_is_off(ctx, dtype):
    """Over all of fp32's range: half of the block's step; that is 1/127 of its largest magnitude from 63.75*2^-126 on; and one
    step, 1/127 of themselves, for magnitudes beyond 127.5*2^121.  (fp32 subtraction of neighbours is exact; so is 64 bits'.)"""
    code, dt = TYPES[dtype]
    top = torch.arange(-149, 128, device="cuda").repeat_interleave(8)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.rand((len(top), 64), generator=g, device="cuda", dtype=torch.float64) * 2 - 1
    x[:, ::32] = 1 + torch.rand((len(top), 2), generator=g, device="cuda", dtype=torch.float64)
    x[::8, 0], x[1::8, 0], x[2::8, 0] = 2.0 - 2.0 ** -8, 127.5 / 64, 127.0 / 64
    x = (x * kept.power(top)[:, None]).to(dt)
    x = torch.where(torch.isfinite(x), x, torch.full_like(x, torch.finfo(dt).max))
    rows, d = x.shape
    ckpt = stored(ctx, x)
    y = torch.empty_like(x)
    dk.dk_ckpt8_load(ctx, dk.dk_ckpt8(rows, d, code), ckpt, y)
    step = kept.power(kept.parts(ckpt, rows, d)[1].to(torch.int64) - 127).repeat_interleave(32, dim=1)
    v, off = x.double(), (y.double() - x.double()).abs()
    largest = v.abs().reshape(rows, -1, 32).amax(dim=2).repeat_interleave(32, dim=1)
    far = v.abs() > 127.5 * 2.0 ** 121
    assert bool(far.any()) == (dtype == "f32")             # (the largest bf16 number is 127.5*2^121)
    assert bool((largest < 63.75 * 2.0 ** -126).any())
    assert bool((off[~far] <= step[~far] / 2).all())
    assert bool((off[far] < step[far]).all()) and bool((off[far] < v[far].abs() / 127).all())
    ordinary = (largest >= 63.75 * 2.0 ** -126) & ~far
    assert bool((off[ordinary] <= largest[ordinary] / 127).all())
    small = largest < 63.75 * 2.0 ** -126
    assert bool((off[small] <= 2.0 ** -127).all()) and not bool(y[v.abs() <= 2.0 ** -127].any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", [(64, 512, 256), (1024, 512, 384), (16384, 1024, 1024), (2047, 1001, 1502), (33000, 40, 24),
                                        (256, 5000, 4096), (4000, 2560, 2560)])
def test_wgrad_sums_of_one_sign(ctx, rows, d, out, dtype):
    """Where the tensor pipe's truncation is a bias.  A promotion every 16 stages of 64 rows (fp32: 4 stages, each of two products)
    is one rounding of 2^-24; each of the 4 instructions of a stage and product before it loses two units of 2^-23 at most of a
    sum that grows to S; the compensation gives back 1.2 (fp32 2.4) times 2^-24 of it for each stage of a chunk; joins of slices,
    undone powers of two and `scale` are 8 roundings more.  fp32: 2^-22 of dy's terms."""
    code, dt = TYPES[dtype]
    x, dy = stored(ctx, draw(rows, d, dt, spread=0.3).abs()), draw(rows, out, dt, seed=5, spread=0.3).abs()
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW = torch.full((out, d), float("nan"), device="cuda")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, dW, None)
    want = dy.double().t() @ kept.decode(x, rows, d)
    stages, chunk, products = -(-rows // 64), 16 if dtype == "bf16" else 4, 1 if dtype == "bf16" else 2
    units = 2 * 4 * products * min(chunk, stages) + 1.2 * products * min(chunk, stages) / 2 + (stages / chunk + 8) / 2
    if dtype == "f32":
        units += 2
    assert bool(((dW.double() - want).abs() <= want * units * 2.0 ** -23).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_wgrad_rows_past_32_bits_of_offset(ctx, dtype):
    """More than 2^31 values of dy and codes of x: sums of small whole numbers, exact but for the compensation (2^-19 of a chunk's
    sum); the rows are zeros but for the first and the last."""
    code, dt = TYPES[dtype]
    rows, d, out, some = 4300000, 500, 504, 1000
    g = torch.Generator(device="cuda").manual_seed(2)
    ends = [torch.randint(-9, 10, (2 * some, n), generator=g, device="cuda").to(dt) for n in (d, out)]
    x, dy = torch.zeros((rows, d), dtype=dt, device="cuda"), torch.zeros((rows, out), dtype=dt, device="cuda")
    for big, small in zip((x, dy), ends):
        big[:some], big[-some:] = small[:some], small[some:]
    ckpt = stored(ctx, x)
    del x
    q = dk.dk_wgrad8(rows, d, out, code)
    ctx.ensure_workspace(q)
    dW, db = torch.empty((out, d), device="cuda"), torch.empty(out, device="cuda")
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, ckpt, 1.0, 0.0, dW, db)
    xv, dyv = ends[0].double(), ends[1].double()
    size = dyv.abs().t() @ xv.abs()
    assert bool(((dW.double() - dyv.t() @ xv).abs() <= size * 2.0 ** -18).all())
    assert torch.equal(db.double(), dyv.sum(dim=0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", [(64, 512, 1000), (300, 333, 77), (256, 1056, 8192), (33000, 40, 24), (2000, 1000, 3001)])
def test_wgrad_tensors_on_any_16_bytes(ctx, rows, d, out, dtype):
    code, dt = TYPES[dtype]

    def shifted(t):
        skip = 16 // t.element_size()
        return torch.empty(t.numel() + skip, dtype=t.dtype, device="cuda")[skip:].view(t.shape).copy_(t)

    x, dy = draw(rows, d, dt, spread=0.5), draw(rows, out, dt, seed=5, spread=0.5)
    ckpt, q, k = stored(ctx, x), dk.dk_wgrad8(rows, d, out, code), dk.dk_ckpt8(rows, d, code)
    ctx.ensure_workspace(q)
    kept_there = shifted(ckpt).zero_()
    dk.dk_ckpt8_store(ctx, k, shifted(x), kept_there)
    assert torch.equal(kept_there, ckpt)
    back = [torch.empty_like(x), shifted(x).zero_()]
    for c, t in zip((ckpt, kept_there), back):
        dk.dk_ckpt8_load(ctx, k, c, t)
    assert torch.equal(*back)
    res = []
    for c, y in ((ckpt, dy), (kept_there, shifted(dy))):
        dW, db = torch.ones((out, d), device="cuda"), torch.ones(out, device="cuda")
        if res:
            dW, db = shifted(dW), shifted(db)
        for keep in (0.0, 0.5):
            dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, y, c, 1.0, keep, dW, db)
        res.append((dW, db))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
