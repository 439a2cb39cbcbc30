"""What the operators around the masked products are measured on: group normalisation with its activation, the
linear layer with softmax cross entropy, and the orthogonalised update.

Together they are the steps of a training pass that the masked products do not cover: a virtual batch holds inputs
of different owners, so the normalisation between two masked layers works on each sample by itself; the loss at the
end produces the first output gradient; the update consumes the decoded weight gradient.

``own`` false: plain torch operations in 32 bits, rounded once at the end.  ``own`` true: the library's calls.
"""
import math

import torch

own = False

COEFS = (3.4445, -4.7750, 2.0315)      # quintic Newton-Schulz polynomial of the orthogonalised update
EPS_NORM, EPS_ORTHO = 1e-5, 1e-7
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one virtual batch (K = 4) of the last ResNet-18 stage: latency
        _norm("norm_fwd_one_virtual_batch", "norm_fwd", 4, 7, 7, 512, 32, "relu", "f32"),
        # sixteen virtual batches of VGG-16's first block at 224x224, activations kept in 16 bits
        _norm("norm_fwd_vgg_block1_bf16", "norm_fwd", 64, 224, 224, 64, 8, "silu", "bf16"),
        # backward of a ResNet-18 stage at its configuration's batch
        _norm("norm_bwd_resnet_stage1", "norm_bwd", 64, 56, 56, 64, 32, "relu", "f32"),
        # odd image and channels that fill no vector of 16 bytes
        _norm("norm_bwd_odd_bf16", "norm_bwd", 27, 37, 53, 60, 5, "silu", "bf16"),
        # scoring with VGG-16's classifier at its configuration's batch: every row's loss, no gradient
        _xent("xent_score_vgg_head", "xent_fwd", 256, 4096, 1000, "f32"),
        # ResNet-18's classifier, one training step at its batch: small, latency counts
        _xent("xent_step_resnet_head", "xent_step", 64, 512, 1000, "f32"),
        # a vocabulary that no tile divides
        _xent("xent_step_odd_vocabulary_bf16", "xent_step", 2047, 1024, 50257, "bf16"),
        # the largest: a long batch of tokens on a large vocabulary
        _xent("xent_step_large_bf16", "xent_step", 4096, 4096, 128000, "bf16"),
        # the update of VGG-16's conv1_2 (64 filters of 3x3x64)
        _ortho("ortho_conv1_2", 1, 64, 576, "f32"),
        # the three 512-channel layers conv4_2, conv4_3 and conv5_1 at once
        _ortho("ortho_three_conv4", 3, 512, 4608, "f32"),
        # a tall weight with odd sizes, gradient in 16 bits
        _ortho("ortho_tall_odd_bf16", 1, 1961, 1001, "bf16"),
        # VGG-16's fc6, the largest weight of the benchmark
        _ortho("ortho_fc6", 1, 4096, 25088, "f32"),
    ]


def _norm(name, op, n, h, w, c, groups, act, dtype):
    return {"name": name, "op": op, "n": n, "h": h, "w": w, "c": c, "groups": groups, "act": act, "dtype": dtype}


def _xent(name, op, rows, d, vocab, dtype):
    return {"name": name, "op": op, "rows": rows, "d": d, "vocab": vocab, "dtype": dtype}


def _ortho(name, batch, m, n, dtype):
    return {"name": name, "op": "ortho", "batch": batch, "m": m, "n": n, "dtype": dtype}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "xent_fwd", "xent_step", "ortho", "ortho"])
    dtype = rng.choice(["f32", "bf16"])
    most = [c for c in listed() if c["op"] == op or (op == "xent_fwd" and c["op"] == "xent_step")
            or (op == "norm_bwd" and c["op"] == "norm_fwd")]
    top_b, top_f = max(work(c)["bytes"] for c in most), max(work(c)["flops"] for c in most)
    while True:
        if op in ("norm_fwd", "norm_bwd"):
            groups = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
            c = groups * _log(rng, 1, 64)
            case = _norm("", op, _log(rng, 1, 256), _log(rng, 1, 224), _log(rng, 1, 224), c, groups,
                         rng.choice(["none", "relu", "silu"]), dtype)
        elif op in ("xent_fwd", "xent_step"):
            case = _xent("", op, _log(rng, 1, 8192), _log(rng, 16, 4096), _log(rng, 10, 128000), dtype)
        else:
            case = _ortho("", rng.choice([1, 1, 2, 4]), _log(rng, 8, 4096), _log(rng, 8, 25088), dtype)
        w = work(case)
        # sums over thousands of rows need values to sum: an image of one pixel in a group of one channel has none
        if op.startswith("norm") and case["h"] * case["w"] * case["c"] // case["groups"] < 16:
            continue
        if w["bytes"] <= top_b and w["flops"] <= top_f:
            del case["name"]
            return case


def work(case):
    """Bytes: every input read once, every output written once.  Flops: the products of the formulas (a symmetric
    result's half), for the loss with gradient the logits once."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("norm"):
        e = case["n"] * case["h"] * case["w"] * case["c"]
        small = 8 * case["c"] + 8 * case["n"] * case["groups"]
        if case["op"] == "norm_fwd":
            return {"bytes": 2 * e * es + small, "flops": 8 * e}
        return {"bytes": 3 * e * es + 2 * small, "flops": 16 * e}
    if case["op"].startswith("xent"):
        t, d, v = case["rows"], case["d"], case["vocab"]
        if case["op"] == "xent_fwd":
            return {"bytes": (t * d + v * d) * es + 16 * t, "flops": 2 * t * d * v}
        return {"bytes": 2 * (t * d + v * d) * es + 16 * t, "flops": 6 * t * d * v}
    b, m, n = case["batch"], min(case["m"], case["n"]), max(case["m"], case["n"])
    return {"bytes": 2 * b * m * n * es, "flops": 5 * b * (3 * m * m * n + m * m * m)}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {"case": dict(case)}
    if case["op"].startswith("norm"):
        n, h, w, c, groups = (case[k] for k in ("n", "h", "w", "c", "groups"))
        # the decoded outputs of a convolution: each channel has its own mean and spread
        x = normal(n, h, w, c)
        x.mul_(0.5 + torch.rand(c, generator=g, device="cuda")).add_(0.3 + 0.5 * normal(c))
        s["gamma"], s["beta"] = 1.0 + 0.1 * normal(c), 0.1 * normal(c)
        s["x"] = x.to(dt)
        del x
        s["stats"] = torch.empty((n, groups, 2), device="cuda")
        if case["op"] == "norm_fwd":
            s["y"] = torch.empty_like(s["x"])
        else:
            v = s["x"].float().reshape(n, h * w, groups, c // groups)
            mean = v.mean(dim=(1, 3))
            rstd = ((v - mean[:, None, :, None]).square().mean(dim=(1, 3)) + EPS_NORM).rsqrt()
            s["stats"][..., 0], s["stats"][..., 1] = mean, rstd
            if case["act"] == "relu":      # the derivative is not defined at the kink: no value is left beside it
                pre = (v - mean[:, None, :, None]) * rstd[:, None, :, None]
                pre = pre * s["gamma"].reshape(groups, -1) + s["beta"].reshape(groups, -1)
                s["x"] = torch.where(pre.abs().reshape(s["x"].shape) < 1e-4, s["x"] + 0.0625, s["x"])
            s["dy"] = normal(n, h, w, c).to(dt)
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    elif case["op"].startswith("xent"):
        t, d, v = case["rows"], case["d"], case["vocab"]
        W = normal(v, d).mul_(2.0 / math.sqrt(d))
        target = torch.randint(0, v, (t,), generator=g, device="cuda")
        # a partly trained model: the features lean towards their own class, the logits spread over a few units
        h = normal(t, d) + W[target] * (4.0 * torch.rand((t, 1), generator=g, device="cuda") * 0.25)
        ignored = torch.rand(t, generator=g, device="cuda") < 0.03
        ignored[0] = False
        s["target"] = torch.where(ignored, torch.full_like(target, -100), target)
        s["h"], s["W"] = h.to(dt), W.to(dt)
        s["scale"] = 1.0 / t
        s["loss"], s["lse"] = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        if case["op"] == "xent_step":
            s["dh"], s["dW"] = torch.empty_like(s["h"]), torch.empty_like(s["W"])
    else:
        b, m, n = case["batch"], case["m"], case["n"]
        # a gradient: a few strong directions that decay, over a floor of noise
        r = min(m, n, 64)
        decay = torch.exp(-4.0 * torch.arange(r, device="cuda") / r)
        x = (normal(b, m, r) * decay) @ normal(b, r, n) * (1e-3 / math.sqrt(r))
        s["x"] = (x + 5e-4 * normal(b, m, n)).to(dt)
        s["out"] = torch.empty_like(s["x"])
        s["scale"] = math.sqrt(max(1.0, m / n))
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    return _own_run(s) if own else _PLAIN[s["case"]["op"]](s)


_context = []


def _own_run(s):
    from paper_2207_00083_b200 import binding as dk
    c = s["case"]
    if not _context:
        _context.append(dk.Context(0))
    ctx = _context[0]
    dt = dk.DK_F32 if c["dtype"] == "f32" else dk.DK_BF16
    if "q" not in s:
        if c["op"].startswith("norm"):
            act = {"none": dk.DK_ACT_NONE, "relu": dk.DK_ACT_RELU, "silu": dk.DK_ACT_SILU}[c["act"]]
            s["q"] = dk.dk_norm(c["n"], c["h"], c["w"], c["c"], c["groups"], act, dt, EPS_NORM)
        elif c["op"].startswith("xent"):
            s["q"] = dk.dk_xent(c["rows"], c["d"], c["vocab"], dt)
        else:
            s["q"] = dk.dk_ortho(c["batch"], c["m"], c["n"], dt, 5, *COEFS, EPS_ORTHO)
        ctx.ensure_workspace(s["q"])
    q = s["q"]
    if c["op"] == "norm_fwd":
        dk.dk_group_norm_fwd(ctx, q, s["x"], s["gamma"], s["beta"], s["y"], s["stats"])
        return {"y": s["y"], "stats": s["stats"]}
    if c["op"] == "norm_bwd":
        dk.dk_group_norm_bwd(ctx, q, s["dy"], s["x"], s["gamma"], s["beta"], s["stats"], s["dx"], s["dgamma"],
                             s["dbeta"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if c["op"] == "ortho":
        dk.dk_orthogonalize(ctx, q, s["x"], s["scale"], 0.0, s["out"])
        return {"out": s["out"]}
    dk.dk_linear_xent_fwd(ctx, q, s["h"], s["W"], s["target"], s["loss"], s["lse"])
    if c["op"] == "xent_fwd":
        return {"loss": s["loss"], "lse": s["lse"]}
    dk.dk_linear_xent_bwd(ctx, q, s["h"], s["W"], s["target"], s["lse"], None, s["scale"], s["dh"], s["dW"])
    return {"loss": s["loss"], "lse": s["lse"], "dh": s["dh"], "dW": s["dW"]}


def _act(pre, act):
    return pre if act == "none" else torch.relu(pre) if act == "relu" else pre / (1.0 + torch.exp(-pre))


def _act_grad(pre, act):
    if act == "none":
        return torch.ones_like(pre)
    if act == "relu":
        return (pre > 0).to(pre.dtype)
    sig = 1.0 / (1.0 + torch.exp(-pre))
    return sig * (1.0 + pre * (1.0 - sig))


def _plain_norm_fwd(s):
    c = s["case"]
    x = s["x"].float().reshape(c["n"], c["h"] * c["w"], c["groups"], -1)
    mean = x.mean(dim=(1, 3), keepdim=True)
    dev = x - mean
    rstd = 1.0 / torch.sqrt((dev * dev).mean(dim=(1, 3), keepdim=True) + EPS_NORM)
    pre = dev * rstd * s["gamma"].reshape(c["groups"], -1) + s["beta"].reshape(c["groups"], -1)
    y = _act(pre, c["act"]).reshape(s["x"].shape).to(s["x"].dtype)
    return {"y": y, "stats": torch.stack((mean[:, 0, :, 0], rstd[:, 0, :, 0]), dim=-1)}


def _plain_norm_bwd(s):
    c = s["case"]
    shape = (c["n"], c["h"] * c["w"], c["groups"], c["c"] // c["groups"])
    x, dy = s["x"].float().reshape(shape), s["dy"].float().reshape(shape)
    gamma, beta = s["gamma"].reshape(c["groups"], -1), s["beta"].reshape(c["groups"], -1)
    mean, rstd = s["stats"][:, None, :, None, 0], s["stats"][:, None, :, None, 1]
    xhat = (x - mean) * rstd
    dpre = dy * _act_grad(xhat * gamma + beta, c["act"])
    dxhat = dpre * gamma
    dx = rstd * (dxhat - dxhat.mean(dim=(1, 3), keepdim=True) - xhat * (dxhat * xhat).mean(dim=(1, 3), keepdim=True))
    return {"dx": dx.reshape(s["x"].shape).to(s["x"].dtype), "dgamma": (dpre * xhat).sum(dim=(0, 1)).reshape(-1),
            "dbeta": dpre.sum(dim=(0, 1)).reshape(-1)}


def _plain_xent(s):
    h, W, target = s["h"].float(), s["W"].float(), s["target"]
    keep = target >= 0
    at = torch.clamp(target, min=0)[:, None]
    logits = h @ W.t()
    top = logits.max(dim=1, keepdim=True).values
    e = torch.exp(logits - top)
    total = e.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    loss = torch.where(keep, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
    out = {"loss": loss, "lse": torch.where(keep, lse, torch.zeros_like(lse))}
    if s["case"]["op"] == "xent_step":
        p = e / total
        p.scatter_add_(1, at, torch.full_like(at, -1, dtype=p.dtype))
        p = p * (keep[:, None] * s["scale"])
        out["dh"] = (p @ W).to(s["h"].dtype)
        out["dW"] = (p.t() @ h).to(s["W"].dtype)
    return out


def _plain_ortho(s):
    a, b, c = COEFS
    x = s["x"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / (torch.sqrt((x * x).sum(dim=(1, 2), keepdim=True)) + EPS_ORTHO)
    for _ in range(5):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    if tall:
        x = x.transpose(1, 2)
    return {"out": (s["scale"] * x).to(s["x"].dtype).contiguous()}


_PLAIN = {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "xent_fwd": _plain_xent, "xent_step": _plain_xent,
          "ortho": _plain_ortho}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"].startswith("norm"):
        n, p, k, cg = case["n"], case["h"] * case["w"], case["groups"], case["c"] // case["groups"]
        # one sample at a time, groups first: [k, p * cg]
        gamma, beta = (s[t].to(f64).reshape(k, 1, cg) for t in ("gamma", "beta"))
        first, stats = torch.empty(s["x"].shape, dtype=f64, device="cuda"), torch.empty((n, k, 2), dtype=f64,
                                                                                        device="cuda")
        dgamma, dbeta = torch.zeros((k, cg), dtype=f64, device="cuda"), torch.zeros((k, cg), dtype=f64, device="cuda")
        for i in range(n):
            x = s["x"][i].to(f64).reshape(p, k, cg).transpose(0, 1)
            if case["op"] == "norm_fwd":
                mean = x.sum(dim=(1, 2)) / (p * cg)
                var = (x * x).sum(dim=(1, 2)) / (p * cg) - mean * mean
                rstd = (var + EPS_NORM) ** -0.5
                stats[i, :, 0], stats[i, :, 1] = mean, rstd
            else:
                mean, rstd = s["stats"][i, :, 0].to(f64), s["stats"][i, :, 1].to(f64)
            xhat = (x - mean[:, None, None]) * rstd[:, None, None]
            z = gamma * xhat + beta
            if case["op"] == "norm_fwd":
                r = z if case["act"] == "none" else z.clamp(min=0) if case["act"] == "relu" else z * torch.sigmoid(z)
            else:
                slope = torch.ones_like(z)
                if case["act"] == "relu":
                    slope = torch.where(z > 0, slope, torch.zeros_like(z))
                elif case["act"] == "silu":
                    sig = torch.sigmoid(z)
                    slope = sig + z * sig * torch.sigmoid(-z)
                d = s["dy"][i].to(f64).reshape(p, k, cg).transpose(0, 1) * slope
                dgamma += (d * xhat).sum(dim=1)
                dbeta += d.sum(dim=1)
                d = d * gamma
                m0 = d.sum(dim=(1, 2)) / (p * cg)
                m1 = (d * xhat).sum(dim=(1, 2)) / (p * cg)
                r = (d - m0[:, None, None] - xhat * m1[:, None, None]) * rstd[:, None, None]
            first[i] = r.transpose(0, 1).reshape(case["h"], case["w"], case["c"])
        if case["op"] == "norm_fwd":
            return {"y": first, "stats": stats}
        return {"dx": first, "dgamma": dgamma.reshape(-1), "dbeta": dbeta.reshape(-1)}
    if case["op"].startswith("xent"):
        t, v = case["rows"], case["vocab"]
        W = s["W"].to(f64)
        live = [i for i, y in enumerate(s["target"].tolist()) if y >= 0]
        loss, lse = torch.zeros(t, dtype=f64, device="cuda"), torch.zeros(t, dtype=f64, device="cuda")
        dh, dW = torch.zeros(s["h"].shape, dtype=f64, device="cuda"), torch.zeros(W.shape, dtype=f64, device="cuda")
        for i in range(0, len(live), 1024):
            rows = torch.tensor(live[i:i + 1024], device="cuda")
            h, y = s["h"][rows].to(f64), s["target"][rows]
            z = h @ W.T
            part = torch.logsumexp(z, dim=1)
            lse[rows] = part
            loss[rows] = part - z[torch.arange(len(rows), device="cuda"), y]
            if case["op"] == "xent_step":
                z = torch.exp(z - part[:, None]) - torch.nn.functional.one_hot(y, v)
                z *= s["scale"]
                dh[rows] = z @ W
                dW += z.T @ h
        out = {"loss": loss, "lse": lse}
        if case["op"] == "xent_step":
            out["dh"], out["dW"] = dh, dW
        return out
    out = []
    for x in s["x"].to(f64):
        wide = x if x.shape[0] <= x.shape[1] else x.T
        y = wide / (torch.linalg.norm(wide) + EPS_ORTHO)
        for _ in range(5):
            q = y @ y.T
            y = COEFS[0] * y + COEFS[1] * (q @ y) + COEFS[2] * (q @ (q @ y))
        out.append((y if wide is x else y.T) * s["scale"])
    return {"out": torch.stack(out)}
