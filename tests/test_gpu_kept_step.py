"""Checkpoints and block norms as a program uses them: a step of a residual network through all of them, captured and
replayed, on other streams, from several threads, within the workspace asked for, with every launch counted and every wait
of the weight gradient's products limited."""
import ctypes
import importlib.util
import os
import threading

import pytest
import torch

import kept
from paper_2207_00083_b200 import binding as dk
from test_gpu_ckpt8 import draw, stored, wgrad_bound

pytestmark = pytest.mark.gpu
TYPES = {dk.DK_F32: torch.float32, dk.DK_BF16: torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    c = dk.Context(0)
    yield c
    assert dk.dk_device_status(c) == 0
    c.close()


class Residual:
    """h0 -> norm -> linear -> (norm, gate, scale, sum, norm) -> linear -> (norm, gate, scale, sum) -> loss, fp32."""
    ROWS, D, CLASSES, EPS, KEEP, SCALE = 96, 160, 40, 1e-5, 1.0, 0.6

    def __init__(self, ctx, kind, gates, held, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        T, D = self.ROWS, self.D
        normal = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
        self.ctx, self.held, self.per = ctx, held, T // gates
        self.params = {"W0": normal(D, D) * D ** -0.5, "W1": normal(D, D) * D ** -0.5, "V": normal(self.CLASSES, D) * D ** -0.5}
        for i in range(2):
            self.params.update({f"pre{i}": 1 + 0.1 * normal(D), f"shift{i}": 0.1 * normal(D), f"post{i}": 1 + 0.1 * normal(D),
                                f"gate{i}": 0.7 + 0.3 * normal(gates, D)})
        self.x, self.target = normal(T, D), torch.randint(0, self.CLASSES, (T,), generator=g, device="cuda")
        self.layer = kind == dk.DK_BLOCK_LAYER
        self.q = dk.dk_block(T, D, self.per, kind, dk.DK_F32, self.EPS, self.KEEP, self.SCALE)
        self.wg, self.head = dk.dk_wgrad8(T, D, D, dk.DK_F32), dk.dk_xent(T, D, self.CLASSES, dk.DK_F32)
        self.k8 = dk.dk_ckpt8(T, D, dk.DK_F32)
        # T rows as 16 virtual batches of 4 + 2 encodings, and as 24 of 4 inputs
        fc = lambda G: dk.dk_problem(dk.DK_FC, dk.DK_NHWC, D, D, 1, 1, 1, 1, 1, 0, 4, G, 0, 0.0)      # noqa: E731
        self.fwd, self.bwd = fc(T // 6), fc(T // 4)
        for q in (self.q, self.wg, self.head, self.fwd, self.bwd):
            ctx.ensure_workspace(q)
        self.loss = torch.empty(T, device="cuda")
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        self.grads.update(x=torch.empty_like(self.x), b0=torch.empty(D, device="cuda"), b1=torch.empty(D, device="cuda"))
        # what a step keeps, and what it passes on
        room = lambda: torch.empty((T, D), device="cuda")      # noqa: E731
        self.t = {k: room() for k in ("n0", "u0", "h1", "n1", "u1", "h2", "dh2", "dh1", "du1", "dn1", "dh0", "du0", "dn0")}
        self.kept = {k: torch.empty(dk.dk_ckpt8_bytes(self.k8), dtype=torch.uint8, device="cuda")
                     for k in ("n0", "n1", "h0", "u0", "h1", "u1")}
        self.stats = [torch.empty((T, 4), device="cuda") for _ in range(3)]
        self.lse = torch.empty(T, device="cuda")

    def step(self):
        c, q, p, t, k, g = self.ctx, self.q, self.params, self.t, self.kept, self.grads
        dk.dk_block_norm_fwd(c, q, self.x, None, None, None, p["pre0"], p["shift0"], None, t["n0"], self.stats[0], k["h0"])
        dk.dk_ckpt8_store(c, self.k8, t["n0"], k["n0"])
        dk.dk_linear_fwd(c, self.fwd, p["W0"], t["n0"], t["u0"])
        dk.dk_block_norm_fwd(c, q, self.x, t["u0"], p["gate0"], p["post0"], p["pre1"], p["shift1"], t["h1"], t["n1"],
                             self.stats[1], None, k["u0"])
        dk.dk_ckpt8_store(c, self.k8, t["n1"], k["n1"])
        dk.dk_linear_fwd(c, self.fwd, p["W1"], t["n1"], t["u1"])
        dk.dk_block_norm_fwd(c, q, t["h1"], t["u1"], p["gate1"], p["post1"], None, None, t["h2"], None, self.stats[2], k["h1"],
                             k["u1"])
        dk.dk_linear_xent_fwd(c, self.head, t["h2"], p["V"], self.target, self.loss, self.lse)
        dk.dk_linear_xent_bwd(c, self.head, t["h2"], p["V"], self.target, self.lse, None, 1.0 / self.ROWS, t["dh2"], g["V"])
        back = dk.dk_block_norm_bwd_ckpt8 if self.held else dk.dk_block_norm_bwd
        h0, u0, h1, u1 = (k[n] for n in ("h0", "u0", "h1", "u1")) if self.held else (self.x, t["u0"], t["h1"], t["u1"])
        back(c, q, t["dh2"], None, h1, u1, p["gate1"], p["post1"], None, self.stats[2], t["dh1"], t["du1"], g["gate1"],
             g["post1"], None, None)
        dk.dk_linear_bwd_wgrad_ckpt8(c, self.wg, t["du1"], k["n1"], 1.0, 0.0, g["W1"], g["b1"])
        dk.dk_linear_bwd_dgrad(c, self.bwd, p["W1"], t["du1"], t["dn1"])
        back(c, q, t["dh1"], t["dn1"], h0, u0, p["gate0"], p["post0"], p["pre1"], self.stats[1], t["dh0"], t["du0"], g["gate0"],
             g["post0"], g["pre1"], g["shift1"])
        dk.dk_linear_bwd_wgrad_ckpt8(c, self.wg, t["du0"], k["n0"], 1.0, 0.0, g["W0"], g["b0"])
        dk.dk_linear_bwd_dgrad(c, self.bwd, p["W0"], t["du0"], t["dn0"])
        back(c, q, t["dh0"], t["dn0"], h0, None, None, None, p["pre0"], self.stats[0], g["x"], None, None, None, g["pre0"],
             g["shift0"])

    def exact(self):
        """Loss and gradients by float64 autograd (b0, b1: of the linear layers' absent biases, the sums of du)."""
        p = {k: v.double().requires_grad_(True) for k, v in self.params.items()}
        x = self.x.double().requires_grad_(True)
        b = [torch.zeros(self.D, dtype=torch.float64, device="cuda", requires_grad=True) for _ in range(2)]

        def norm(v):
            v = v - v.mean(dim=1, keepdim=True) if self.layer else v
            return v / (v.square().mean(dim=1, keepdim=True) + self.EPS).sqrt()

        gate = lambda i: p[f"gate{i}"].repeat_interleave(self.per, dim=0)      # noqa: E731
        h1 = self.KEEP * x + self.SCALE * gate(0) * p["post0"] * norm((norm(x) * p["pre0"] + p["shift0"]) @ p["W0"].T + b[0])
        h2 = self.KEEP * h1 + self.SCALE * gate(1) * p["post1"] * norm((norm(h1) * p["pre1"] + p["shift1"]) @ p["W1"].T + b[1])
        loss = torch.nn.functional.cross_entropy(h2 @ p["V"].T, self.target)
        loss.backward()
        return float(loss), {**{k: v.grad for k, v in p.items()}, "x": x.grad, "b0": b[0].grad, "b1": b[1].grad}


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("gates", [1, 8, 96])
@pytest.mark.parametrize("kind", [dk.DK_BLOCK_RMS, dk.DK_BLOCK_LAYER])
def test_step_of_a_residual_network(ctx, kind, gates, held):
    """Gradients against float64 autograd.  What comes from the weights' products alone is off by fp32 roundings (1e-4).  A
    kept value is off by step/sqrt(12) on average, a step at most 1/63.75 of its block's largest of 32, some 3.5 spreads: 1.6 %
    of the spread.  A weight's gradient sums such values with weights that know nothing of the error (twice that: 3.2 %);
    through a block's norms the errors of h^ and u^ meet in every term, three at most (5 %), and the first block's
    gradients have gone through two."""
    net = Residual(ctx, kind, gates, held)
    net.step()
    loss, want = net.exact()
    assert abs(float(net.loss.mean()) - loss) <= 1e-5 * loss
    for k, w in want.items():
        tol = 0.032 if k in ("W0", "W1") else 1e-4
        if held and k != "V":
            tol = 0.10 if k in ("x", "pre0", "shift0", "W0", "b0") else 0.05
        assert float((net.grads[k].double() - w).norm()) <= tol * float(w.norm()) + 1e-7, k


@pytest.mark.parametrize("held", [False, True])
def test_captured_and_replayed(ctx, held):
    """Two steps of one context in a graph each, replayed in turn with inputs that change between; on a stream of their own."""
    nets = [Residual(ctx, dk.DK_BLOCK_LAYER, 8, held, seed=s) for s in (1, 2)]
    graphs, s = [], torch.cuda.Stream()
    for net in nets:
        net.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            net.step()
        graphs.append(graph)
    for turn in range(3):
        for net, graph in zip(nets, graphs):
            net.x.add_(0.1 * (turn + 1))
            net.params["W1"].mul_(1.01)
            net.step()
            want = {k: v.clone() for k, v in net.grads.items()}
            for v in net.grads.values():
                v.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            for k in want:
                assert torch.equal(net.grads[k], want[k]), k
    del graphs


def test_on_another_stream(ctx):
    net = Residual(ctx, dk.DK_BLOCK_RMS, 8, True)
    net.step()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in net.grads.items()}
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for v in net.grads.values():
            v.zero_()
        net.step()
    s.synchronize()
    for k in want:
        assert torch.equal(net.grads[k], want[k]), k


def test_threads_with_a_context_each():
    failures = []

    def work(seed):
        try:
            c = dk.Context(0)
            net = Residual(c, dk.DK_BLOCK_LAYER, (1, 8, 96)[seed], True, seed)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                net.step()
                s.synchronize()
                want = {k: v.clone() for k, v in net.grads.items()}
                for i in range(100):
                    net.step()
                s.synchronize()
                assert all(torch.equal(net.grads[k], want[k]) for k in want)
            c.close()
        except Exception as e:  # noqa: BLE001 (reported below)
            failures.append((seed, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures


GUARD = 64 << 20
CASES = [dk.dk_wgrad8(1, 1, 1, 0), dk.dk_wgrad8(64, 512, 1000, 0), dk.dk_wgrad8(2047, 1001, 1502, 1), dk.dk_wgrad8(4000, 2560, 2560, 0),
         dk.dk_wgrad8(4000, 2560, 2560, 1), dk.dk_wgrad8(33000, 40, 24, 0), dk.dk_wgrad8(33000, 40, 24, 1),
         dk.dk_wgrad8(70, 33, 4001, 0)] + [
    dk.dk_block(rows, d, per, kind, t, 1e-5, 1.0, 0.5)
    for rows, d, per in ((1, 1, 1), (300, 96, 1), (3001, 40, 64), (300, 1030, 7), (777, 4096, 400), (40, 9000, 3), (5, 16384, 5),
                         (2000, 2050, 2000))
    for kind, t in ((0, 0), (1, 1))]


@pytest.mark.parametrize("q", CASES, ids=lambda q: type(q).__name__ + "_" + "_".join(str(getattr(q, f)) for f, _ in q._fields_[:5]))
def test_guard_behind_the_workspace(q):
    ctx = dk.Context(0)
    need = ctx.step_workspace_bytes(q)
    buf = torch.full((need + GUARD + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    off = (-buf.data_ptr()) % 256
    assert dk.lib().dk_set_workspace(ctx.handle, ctypes.c_void_p(buf.data_ptr() + off), need) == 0
    dt = TYPES[q.dtype]
    if isinstance(q, dk.dk_wgrad8):
        x, dy = stored(ctx, draw(q.rows, q.d, dt, spread=0.5)), draw(q.rows, q.out, dt, spread=0.5)
        out = [torch.empty((q.out, q.d), device="cuda"), torch.empty(q.out, device="cuda")]
        dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, *out)
        small = lambda: dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, *out)      # noqa: E731
    else:
        h, u, dho, dn = (draw(q.rows, q.d, dt, seed=i, spread=0.5) for i in range(4))
        gate, vec = torch.ones((-(-q.rows // q.rows_per_gate), q.d), device="cuda"), torch.ones(q.d, device="cuda")
        new = lambda t: torch.empty_like(t)      # noqa: E731
        st, k = torch.empty((q.rows, 4), device="cuda"), [stored(ctx, t) for t in (h, u)]
        ho, n, dh, du, dg, dpo, dpr, ds = new(h), new(h), new(h), new(h), new(gate), new(vec), new(vec), new(vec)
        dk.dk_block_norm_fwd(ctx, q, h, u, gate, vec, vec, vec, ho, n, st)
        for g, d_g in ((gate, dg), (None, None)):
            dk.dk_block_norm_bwd(ctx, q, dho, dn, h, u, g, vec, vec, st, dh, du, d_g, dpo, dpr, ds)
            dk.dk_block_norm_bwd_ckpt8(ctx, q, dho, dn, k[0], k[1], g, vec, vec, st, dh, du, d_g, dpo, dpr, None)
        out = [ho, n, st, dh, du, dg, dpo, dpr, ds]
        small = lambda: dk.dk_block_norm_bwd(ctx, q, dho, dn, h, u, gate, vec, vec, st, dh, du, dg, dpo, dpr, ds)      # noqa: E731
    torch.cuda.synchronize()
    assert all(bool(torch.isfinite(o).all()) for o in out)
    assert bool((buf[off + need:] == 0xA5).all()) and bool((buf[:off] == 0xA5).all())
    assert dk.lib().dk_set_workspace(ctx.handle, ctypes.c_void_p(buf.data_ptr() + off), 0) == 0
    with pytest.raises(dk.DkError) as e:
        small()
    assert e.value.status == 4                                  # DK_ERR_WORKSPACE
    ctx.close()


def count_launches(ctx, call):
    """dk_profile_read counts every kernel that a call launches: as many as the call leaves in a captured graph."""
    call()
    torch.cuda.synchronize()
    dk.dk_profile_reset(ctx)
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    cuda, of, n = ctypes.CDLL("libcuda.so.1"), ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert cuda.cuGraphGetNodes(of, None, ctypes.byref(n)) == 0 and n.value > 0
    nodes, kind = (ctypes.c_void_p * n.value)(), ctypes.c_int()
    assert cuda.cuGraphGetNodes(of, nodes, ctypes.byref(n)) == 0
    kernels = 0
    for node in nodes:
        assert cuda.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        kernels += kind.value == 0                              # CU_GRAPH_NODE_TYPE_KERNEL
    assert kernels and dk.dk_profile_read(ctx)["other"][2] == kernels


# small tiles, pair tiles with and without a cut last wave, slices joined by a kernel of their own
WGRADS = [(64, 512, 1000), (4000, 2560, 2560), (300, 2600, 4100), (33000, 40, 24), (2000, 1000, 3001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", WGRADS)
def test_launches_are_counted(ctx, rows, d, out, dtype):
    q, dt = dk.dk_wgrad8(rows, d, out, dtype), TYPES[dtype]
    ctx.ensure_workspace(q)
    x, dy, dW, db = stored(ctx, draw(rows, d, dt)), draw(rows, out, dt), torch.empty((out, d), device="cuda"), torch.empty(out, device="cuda")
    for b in (db, None):
        count_launches(ctx, lambda: dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, dW, b))


def test_launches_of_the_others_are_counted(ctx):
    k, q = dk.dk_ckpt8(100, 60, dk.DK_F32), dk.dk_block(100, 60, 7, 0, dk.DK_F32, 1e-5, 1.0, 1.0)
    ctx.ensure_workspace(q)
    h, u, gate, vec = draw(100, 60, torch.float32), draw(100, 60, torch.float32), torch.ones((15, 60), device="cuda"), torch.ones(60, device="cuda")
    kh, ku, st = stored(ctx, h), stored(ctx, u), torch.empty((100, 4), device="cuda")
    a, b, dgate, dpost, dpre = (torch.empty_like(t) for t in (h, h, gate, vec, vec))
    count_launches(ctx, lambda: dk.dk_ckpt8_store(ctx, k, h, kh))
    count_launches(ctx, lambda: dk.dk_ckpt8_load(ctx, k, kh, a))
    count_launches(ctx, lambda: dk.dk_block_norm_fwd(ctx, q, h, u, gate, vec, vec, None, a, b, st, kh, ku))
    count_launches(ctx, lambda: dk.dk_block_norm_bwd_ckpt8(ctx, q, h, u, kh, ku, gate, vec, vec, st, a, b, dgate, dpost, dpre,
                                                           None))
    for c, groups in ((64, 8), (60, 5)):                        # (the checkpoint with the values, and by itself)
        for n, hw in ((3, 5), (4, 200)):
            x, g = draw(n * hw * hw, c, torch.float32), torch.ones(c, device="cuda")
            qn, ck = dk.dk_norm(n, hw, hw, c, groups, 2, dk.DK_F32, 1e-5), stored(ctx, x)
            ctx.ensure_workspace(qn)
            y, s, dg, db = torch.empty_like(x), torch.empty((n, groups, 2), device="cuda"), torch.empty_like(g), torch.empty_like(g)
            count_launches(ctx, lambda: dk.dk_group_norm_fwd_ckpt8(ctx, qn, x, g, g, y, s, ck))
            count_launches(ctx, lambda: dk.dk_group_norm_bwd_ckpt8(ctx, qn, x, ck, g, g, s, y, dg, db))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,d,out", WGRADS)
def test_waits_of_the_weight_gradient(ctx, rows, d, out, dtype):
    """A producer arms a stage without copying (a host-set option): the call ends, the status says so, and the next call, whose
    counters dk_device_status has cleared, is as it should be."""
    q, dt = dk.dk_wgrad8(rows, d, out, dtype), TYPES[dtype]
    ctx.ensure_workspace(q)
    x, dy = stored(ctx, draw(rows, d, dt, spread=0.5)), draw(rows, out, dt, spread=0.5)
    dW, db = torch.empty((out, d), device="cuda"), torch.empty(out, device="cuda")
    dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 12)
    dk.dk_set_option(ctx, dk.DK_OPT_TEST_WITHHOLD, 0)
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, dW, db)
    assert dk.dk_device_status(ctx) == dk.DK_ERR_TIMEOUT and dk.dk_device_status(ctx) == 0
    dk.dk_set_option(ctx, dk.DK_OPT_SPIN_LIMIT, 1 << 22)
    dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, dy, x, 1.0, 0.0, dW, db)
    xv, dyv = kept.decode(x, rows, d), dy.double()
    assert bool(((dW.double() - dyv.t() @ xv).abs() <= wgrad_bound(dyv, xv, "f32" if dtype == dk.DK_F32 else "bf16")).all())
    assert dk.dk_device_status(ctx) == 0


def test_example_with_kept_inputs():
    """The example's gradients with its norms' inputs kept in 8 bits, against those with them kept as they are: 1.6 % of the
    inputs' spread, in every term of a norm's backward pass (5 %), after one norm or two (10 %)."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "masked_training.py")
    spec = importlib.util.spec_from_file_location("masked_training", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    out = []
    for keep8 in (False, True):
        net = m.Network(seed=3, keep8=keep8)
        x, target = next(m.images(net.n, seed=4))
        out.append(net.gradients(x, target))
        assert dk.dk_device_status(net.ctx) == 0
        net.ctx.close()
    assert abs(float(out[0][0]) - float(out[1][0])) <= 1e-3 * float(out[0][0])
    for k, g in out[0][1].items():
        tol = 1e-3 if k == "V" else 0.05 if k.endswith("1") else 0.10
        assert float((out[1][1][k] - g).norm()) <= tol * float(g.norm()), k
