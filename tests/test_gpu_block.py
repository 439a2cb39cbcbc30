"""The norms before and after a residual block with its gate and residual scale, against the formulas in 64 bits."""
import pytest
import torch

import kept
from paper_2207_00083_b200 import binding as dk

pytestmark = pytest.mark.gpu
TYPES = {"f32": (dk.DK_F32, torch.float32), "bf16": (dk.DK_BF16, torch.bfloat16)}
EPS, KEEP, SCALE = 1e-5, 0.9, 0.7
# Roundings of 2^-24 on the way to a value, relative to the magnitudes it is formed from.  A norm: a sum over a row is at
# most 16 additions in a thread, 5 in a warp, 5 over warps, twice with the mean; some 8 more for the division, root and
# products; two norms one after the other, and half of that again for the gradients' own sums.
FWD, BWD = 96 * 2.0 ** -24, 192 * 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    assert dk.dk_device_status(c) == 0
    c.close()


class Case:
    def __init__(self, rows, d, kind="rms", gate="none", per=1, dtype="f32", branch=True, norm=True, shift=False, dh=True,
                 seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + 13 * rows + d)
        self.code, self.dt = TYPES[dtype]
        self.rows, self.d, self.layer, self.per = rows, d, kind == "layer", rows if gate == "channel" else per

        def normal(*shape):
            return torch.randn(shape, generator=g, device="cuda")

        def tensor():
            return (normal(rows, d) * torch.exp(0.5 * normal(d)) + 0.5 * normal(d)).to(self.dt)

        gates = 0 if gate == "none" or not branch else -(-rows // self.per)
        self.h, self.u = tensor(), tensor() if branch else None
        self.gate = normal(gates, d) if gates else None
        self.post = 1 + 0.2 * normal(d) if branch else None
        self.pre = 1 + 0.2 * normal(d) if norm else None
        self.shift = 0.3 * normal(d) if shift and norm else None
        self.dh_out = tensor() if dh else None
        self.dn = tensor() if norm else None
        self.q = dk.dk_block(rows, d, max(1, self.per), dk.DK_BLOCK_LAYER if self.layer else dk.DK_BLOCK_RMS, self.code, EPS,
                             KEEP, SCALE)

    def forward(self, ctx, checkpoints=True, stats=True):
        new = lambda t: torch.full_like(t, float("nan"))      # noqa: E731
        self.h_out = new(self.h) if self.u is not None else None
        self.n = new(self.h) if self.pre is not None else None
        self.stats = torch.full((self.rows, 4), float("nan"), device="cuda") if stats else None
        self.kh, self.ku = (torch.full((kept.size(self.rows, self.d),), 0xAB, dtype=torch.uint8, device="cuda")
                            if checkpoints and t is not None else None for t in (self.h, self.u))
        dk.dk_block_norm_fwd(ctx, self.q, self.h, self.u, self.gate, self.post, self.pre, self.shift, self.h_out, self.n,
                             self.stats, self.kh, self.ku)

    def backward(self, ctx, held):
        new = lambda t: None if t is None else torch.full_like(t, float("nan"))      # noqa: E731
        out = {"dh": new(self.h), "du": new(self.u), "dgate": new(self.gate), "dpost": new(self.post), "dpre": new(self.pre),
               "dshift": new(self.shift)}
        call, h, u = (dk.dk_block_norm_bwd_ckpt8, self.kh, self.ku) if held else (dk.dk_block_norm_bwd, self.h, self.u)
        call(ctx, self.q, self.dh_out, self.dn, h, u, self.gate, self.post, self.pre, self.stats, *out.values())
        return out

    # ---- 64 bits: values, and the magnitudes they are formed from ----
    def moments(self, x, mag):
        """mean, 1/sqrt(..), and the magnitude of the normalised values' error"""
        mean = x.mean(dim=1, keepdim=True) if self.layer else torch.zeros_like(x[:, :1])
        r = 1 / (((x - mean) ** 2).mean(dim=1, keepdim=True) + EPS).sqrt()
        hat = (x - mean) * r
        return mean, r, hat, (mag + mag.mean(dim=1, keepdim=True)) * r + hat.abs() * (1 + ((mag * r) * hat.abs()).mean(dim=1, keepdim=True))

    def gates(self):
        if self.gate is None:
            return torch.ones((1, 1), dtype=torch.float64, device="cuda")
        return self.gate.double()[torch.arange(self.rows, device="cuda") // self.per]

    def want_forward(self):
        w, m = {}, {}
        h = self.h.double()
        s, mag = h, h.abs()
        stats = torch.zeros((self.rows, 4), dtype=torch.float64, device="cuda")
        stat_mag = torch.zeros_like(stats)
        if self.u is not None:
            u = self.u.double()
            mu, ru, uh, um = self.moments(u, u.abs())
            f = SCALE * self.gates() * self.post.double()
            s, mag = KEEP * h + f * uh, KEEP * h.abs() + f.abs() * um
            stats[:, :1], stats[:, 1:2] = mu, ru
            stat_mag[:, :1], stat_mag[:, 1:2] = u.abs().mean(dim=1, keepdim=True), ru * (1 + (u.abs() * ru * uh.abs()).mean(dim=1, keepdim=True))
            w["h_out"], m["h_out"] = s, mag
        if self.pre is not None:
            mh, rh, hh, hm = self.moments(s, mag)
            w["n"], m["n"] = hh * self.pre.double(), hm * self.pre.double().abs()
            if self.shift is not None:
                w["n"], m["n"] = w["n"] + self.shift.double(), m["n"] + self.shift.double().abs()
            stats[:, 2:3], stats[:, 3:] = mh, rh
            stat_mag[:, 2:3], stat_mag[:, 3:] = mag.mean(dim=1, keepdim=True), rh * (1 + (mag * rh * hh.abs()).mean(dim=1, keepdim=True))
        w["stats"], m["stats"] = stats, stat_mag
        return w, m

    def want_backward(self, h, u):
        """From h and u as given, with the forward call's statistics."""
        w, m = {}, {}
        mu, ru, mh, rh = (self.stats.double()[:, i:i + 1] for i in range(4))
        D = torch.zeros_like(h) if self.dh_out is None else self.dh_out.double()
        Dm = D.abs()
        if u is not None:
            uh, um = (u - mu) * ru, (u.abs() + mu.abs()) * ru
            f = SCALE * self.gates() * self.post.double()
            s, mag = KEEP * h + f * uh, KEEP * h.abs() + f.abs() * um
        else:
            s, mag = h, h.abs()
        mean = lambda t: t.mean(dim=1, keepdim=True)      # noqa: E731
        if self.pre is not None:
            hh, hm = (s - mh) * rh, (mag + mh.abs()) * rh
            dn = self.dn.double()
            q = dn * self.pre.double()
            D = D + rh * (q - (mean(q) if self.layer else 0) - hh * mean(q * hh))
            Dm = Dm + rh * (q.abs() + (mean(q.abs()) if self.layer else 0) + hm * mean((q * hh).abs()) + hh.abs() * mean(q.abs() * hm))
            w["dpre"], m["dpre"] = (dn * hh).sum(dim=0), (dn.abs() * hm).sum(dim=0)
            w["dshift"], m["dshift"] = dn.sum(dim=0), dn.abs().sum(dim=0)
        w["dh"], m["dh"] = (KEEP * D, KEEP * Dm) if u is not None else (D, Dm)
        if u is not None:
            s, sm = f * D, f.abs() * Dm
            w["du"] = ru * (s - (mean(s) if self.layer else 0) - uh * mean(s * uh))
            m["du"] = ru * (sm + (mean(sm) if self.layer else 0) + um * mean(sm * uh.abs()) + uh.abs() * mean(sm * um))
            E, Em = SCALE * D * uh, SCALE * Dm * (uh.abs() + um)
            w["dpost"], m["dpost"] = (E * self.gates()).sum(dim=0), (Em * self.gates().abs()).sum(dim=0)
            if self.gate is not None:
                row = torch.arange(self.rows, device="cuda") // self.per
                zero = torch.zeros(self.gate.shape, dtype=torch.float64, device="cuda")
                w["dgate"] = zero.index_add(0, row, E * self.post.double())
                m["dgate"] = zero.index_add(0, row, Em * self.post.double().abs())
        return w, m

    def check_forward(self, ctx):
        self.forward(ctx)
        w, m = self.want_forward()
        near(self.h_out, "h_out", w, m, FWD)
        near(self.n, "n", w, m, FWD)
        near(self.stats, "stats", w, m, FWD)
        for t, k in ((self.h, self.kh), (self.u, self.ku)):
            if t is not None:
                assert torch.equal(k, kept.pack(*kept.encode(t)))

    def check_backward(self, ctx, held):
        got = self.backward(ctx, held)
        h, u = (None if t is None else kept.decode(k, self.rows, self.d) if held else t.double()
                for t, k in ((self.h, self.kh), (self.u, self.ku)))
        w, m = self.want_backward(h, u)
        # (sums over rows: a team's, then at most 1024 parts by sixteen)
        far = BWD + 2.0 ** -24 * (self.rows / 148 + 128)
        for k, t in got.items():
            near(t, k, w, m, BWD if k in ("dh", "du") else far)
        return got


def near(got, name, want, mag, units):
    if got is None:
        return
    w, tol = want[name], mag[name] * units + 1e-37
    if got.dtype == torch.bfloat16:
        tol = tol + (w.abs() + tol) * 2.0 ** -8
    err = (got.double() - w).abs()
    assert bool((err <= tol).all()), (name, float((err / tol).max()))


SHAPES = [(1, 1), (1, 32), (2, 33), (5, 60), (3, 100), (130, 34), (67, 256), (40, 257), (9, 1001), (300, 512), (7, 2050), (2, 4096),
          (3, 4100), (5, 8192), (2, 8200), (3, 16384), (2, 16383), (2000, 64), (1111, 129), (700, 1024)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("rows,d", SHAPES)
def test_both_directions(ctx, rows, d, kind, dtype):
    c = Case(rows, d, kind, "channel", 1, dtype, shift=kind == "layer")
    ctx.ensure_workspace(c.q)
    c.check_forward(ctx)
    c.check_backward(ctx, False)
    c.check_backward(ctx, True)


GATES = [("none", 1), ("channel", 1), ("rows", 1), ("rows", 3), ("rows", 64), ("rows", 299), ("rows", 300), ("rows", 5000)]


@pytest.mark.parametrize("gate,per", GATES)
@pytest.mark.parametrize("rows,d,kind,dtype", [(300, 96, "layer", "f32"), (300, 1030, "rms", "bf16"), (300, 520, "layer", "bf16"),
                                               (3001, 40, "rms", "f32"), (3001, 1001, "layer", "f32"), (40, 9000, "rms", "f32")])
def test_gates(ctx, rows, d, kind, dtype, gate, per):
    c = Case(rows, d, kind, gate, per, dtype)
    ctx.ensure_workspace(c.q)
    c.check_forward(ctx)
    for held in (False, True):
        c.check_backward(ctx, held)


@pytest.mark.parametrize("d", [64, 1001, 10000])
@pytest.mark.parametrize("branch,norm,dh", [(False, True, True), (False, True, False), (True, False, True), (True, True, False)])
def test_parts_of_it(ctx, d, branch, norm, dh):
    """Before the first block, after the last one, and without a gradient of the sum."""
    c = Case(37, d, "layer", "rows", 5, "bf16", branch=branch, norm=norm, dh=dh, shift=True)
    ctx.ensure_workspace(c.q)
    c.check_forward(ctx)
    for held in (False, True):
        c.check_backward(ctx, held)


@pytest.mark.parametrize("d", [96, 1001, 5000])
def test_in_place(ctx, d):
    """h_out over h and dh over dh_out; without statistics and checkpoints; the same bits again and again."""
    c = Case(50, d, "layer", "channel", 1, "bf16", shift=True)
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    got = c.backward(ctx, True)
    h, n = c.h.clone(), torch.empty_like(c.n)
    dk.dk_block_norm_fwd(ctx, c.q, h, c.u, c.gate, c.post, c.pre, c.shift, h, n, None)
    assert torch.equal(h, c.h_out) and torch.equal(n, c.n)
    again = {k: torch.empty_like(t) for k, t in got.items()}
    over = c.dh_out.clone()
    dk.dk_block_norm_bwd_ckpt8(ctx, c.q, over, c.dn, c.kh, c.ku, c.gate, c.post, c.pre, c.stats, over, again["du"], again["dgate"],
                               again["dpost"], again["dpre"], again["dshift"])
    again["dh"] = over
    for k in got:
        assert torch.equal(again[k], got[k]), k


def test_nothing(ctx):
    c = Case(0, 40, "layer", "none", 1, "f32", shift=True)
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    got = c.backward(ctx, False)
    for k in ("dpost", "dpre", "dshift"):
        assert not bool(got[k].any()) and bool(torch.isfinite(got[k]).all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_one_value_and_infinities(ctx, kind):
    """A row of zeros and one of a single value are finite with eps > 0; an infinity or a NaN stays in its own row."""
    c = Case(8, 200, kind, "none", 1, "f32")
    c.h[1], c.u[1], c.u[2], c.u[3, 5], c.h[4, 7] = 0.0, 0.0, 3.0, float("inf"), float("nan")
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    bad = [3, 4]
    for t in (c.h_out, c.n):
        rows = torch.isfinite(t).all(dim=1)
        assert (~torch.isfinite(c.n).all(dim=1)).nonzero().flatten().tolist() == bad
        assert bool(rows[[0, 1, 2, 5, 6, 7]].all())
    got = c.backward(ctx, False)
    ok = [i for i in range(8) if i not in bad]
    assert bool(torch.isfinite(got["dh"][ok]).all()) and bool(torch.isfinite(got["du"][ok]).all())


@pytest.mark.parametrize("d,dtype", [(4096, "bf16"), (1001, "f32"), (512, "bf16"), (300, "f32")])
@pytest.mark.parametrize("row", [0, 1, 2])
def test_copies_that_do_not_come(ctx, d, dtype, row):
    """A host-set option makes the first team arm a row without copying it (a team of 512 values has five of these rows, the
    others more): every wait ends within a short poll limit, the
    status says so, and the next call is as it should be."""
    c = Case(12000, d, "rms", "channel", 1, dtype)
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    for held in (None, False, True):
        dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 12)
        dk.dk_set_option(ctx, dk.DK_OPT_TEST_WITHHOLD, row)
        if held is None:
            c.forward(ctx, checkpoints=False, stats=False)
        else:
            c.backward(ctx, held)
        assert dk.dk_get_option(ctx, dk.DK_OPT_TEST_WITHHOLD) == -1
        assert dk.dk_device_status(ctx) == dk.DK_ERR_TIMEOUT
        assert dk.dk_device_status(ctx) == 0
        dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 22)
        c.check_forward(ctx)
        c.check_backward(ctx, bool(held))


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_against_differences(ctx, kind):
    """Slopes of <h_out, a> + <n, b> along a random direction of every input, from the forward call itself: its rounding
    (2^-24 of some hundred terms over a step of 1/64) and the step's third derivative leave under 1e-3 of the slope's
    scale."""
    c = Case(24, 96, kind, "rows", 5, "f32", shift=True)
    ctx.ensure_workspace(c.q)
    c.forward(ctx)
    got = c.backward(ctx, False)
    value = lambda: float((c.h_out.double() * c.dh_out.double()).sum() + (c.n.double() * c.dn.double()).sum())      # noqa: E731
    for name in ("h", "u", "gate", "post", "pre", "shift"):
        t = getattr(c, name)
        v = torch.randn(t.shape, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
        base, step, at = t.clone(), 1 / 64, []
        for sign in (1, -1):
            setattr(c, name, base + sign * step * v)
            c.forward(ctx, checkpoints=False, stats=False)
            at.append(value())
        setattr(c, name, base)
        slope = (at[0] - at[1]) / (2 * step)
        want = float((got["d" + name].double() * v.double()).sum())
        scale = float((got["d" + name].double().norm() * v.double().norm()))
        assert abs(slope - want) <= 1e-3 * scale, name
