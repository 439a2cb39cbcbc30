"""What the 8-bit activation checkpoints, their use in the backward pass, and the norms before and after a residual block
are measured on.

A training step keeps every layer's input from the forward to the backward pass.  ``ckpt`` holds such a tensor in 8 bits
(whole numbers of 8 bits under a power of two for each 32 values of a row) and brings it back; ``norm_step`` is a group
normalisation whose input is kept like that, forward and backward; ``wgrad`` is the weight gradient of a linear layer from
its kept input.  ``block_fwd`` and ``block_step`` are what lies between two residual blocks: the norm after the one, its
gate and residual scale, the sum, and the norm before the next.

``own`` false: plain torch operations in 32 bits, rounded once at the end.  ``own`` true: the library's calls.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 32                             # values of a row that share a power of two
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one virtual batch (K = 4) of the last ResNet-18 stage, kept and brought back: latency
        _ckpt("ckpt_one_virtual_batch", 196, 512, "f32"),
        # sixteen virtual batches of VGG-16's first block at 224x224, channels-last, in 16 bits
        _ckpt("ckpt_vgg_block1_bf16", 64 * 224 * 224, 64, "bf16"),
        # a ResNet-18 stage at its configuration's batch, both directions
        _norm("norm_step_resnet_stage1", 64, 56, 56, 64, 32, "none", "f32"),
        # odd image, channels that fill neither a vector of 16 bytes nor the last 32 values
        _norm("norm_step_odd_bf16", 27, 37, 53, 60, 5, "silu", "bf16"),
        # ResNet-18's classifier at its batch: small, latency counts
        _wgrad("wgrad_resnet_head", 64, 512, 1000, "f32"),
        # VGG-16's fc6, the largest weight of the benchmark, at its batch
        _wgrad("wgrad_fc6", 256, 25088, 4096, "f32"),
        # a long batch of tokens through a wide layer
        _wgrad("wgrad_large_bf16", 16384, 4096, 4096, "bf16"),
        # rows and features that no tile divides
        _wgrad("wgrad_odd_bf16", 2047, 1001, 1502, "bf16"),
        # one token between two blocks of a model that answers: latency
        _block("block_fwd_one_token_bf16", "block_fwd", 1, 4096, "rms", "channel", 1, 0, "bf16"),
        # a prompt, rows of no whole vectors
        _block("block_fwd_odd", "block_fwd", 2047, 1001, "layer", "none", 1, 0, "f32"),
        # a training step, one gate a sample, inputs kept in 8 bits: the largest
        _block("block_step_kept_bf16", "block_step", 16384, 4096, "rms", "rows", 2048, 1, "bf16"),
        # the same with a learned gate and the inputs kept as they are, in 32 bits
        _block("block_step_f32", "block_step", 4095, 2050, "layer", "channel", 1, 0, "f32"),
    ]


def _ckpt(name, rows, d, dtype):
    return {"name": name, "op": "ckpt", "rows": rows, "d": d, "dtype": dtype}


def _norm(name, n, h, w, c, groups, act, dtype):
    return {"name": name, "op": "norm_step", "n": n, "h": h, "w": w, "c": c, "groups": groups, "act": act, "dtype": dtype}


def _wgrad(name, rows, d, out, dtype):
    return {"name": name, "op": "wgrad", "rows": rows, "d": d, "out": out, "dtype": dtype}


def _block(name, op, rows, d, kind, gate, per, kept, dtype):
    """gate: none, channel (one for all rows), rows (one for each `per` rows); kept: inputs held in 8 bits."""
    return {"name": name, "op": op, "rows": rows, "d": d, "kind": kind, "gate": gate, "per": per, "kept": bool(kept),
            "dtype": dtype}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ckpt", "norm_step", "wgrad", "wgrad", "block_fwd", "block_step", "block_step"])
    dtype = rng.choice(["f32", "bf16"])
    of = [c for c in listed() if c["op"] in (op, "block_step" if op == "block_fwd" else op)]
    top_b, top_f = max(work(c)["bytes"] for c in of), max(work(c)["flops"] for c in of)
    while True:
        if op == "ckpt":
            case = _ckpt("", _log(rng, 1, 1 << 20), _log(rng, 8, 16384), dtype)
        elif op == "norm_step":
            groups = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
            case = _norm("", _log(rng, 1, 256), _log(rng, 1, 224), _log(rng, 1, 224), groups * _log(rng, 1, 64), groups,
                         rng.choice(["none", "silu"]), dtype)
            # sums over thousands of rows need values to sum
            if case["h"] * case["w"] * case["c"] // groups < 16:
                continue
        elif op == "wgrad":
            case = _wgrad("", _log(rng, 1, 32768), _log(rng, 16, 25088), _log(rng, 16, 8192), dtype)
        else:
            gate = rng.choice(["none", "channel", "rows"])
            rows = _log(rng, 1, 65536)
            case = _block("", op, rows, _log(rng, 32, 8192), rng.choice(["rms", "layer"]), gate,
                          _log(rng, 1, rows) if gate == "rows" else 1, op == "block_step" and rng.random() < 0.6, dtype)
        w = work(case)
        if w["bytes"] <= top_b and w["flops"] <= top_f:
            del case["name"]
            return case


def _padded(d):
    return -(-d // BLOCK) * BLOCK


def work(case):
    """Bytes: every input read once, every output written once; what is held in 8 bits between the two directions is
    written once and read once.  Flops: the product of the formula; of the others the operations of a value."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "ckpt":
        e = case["rows"] * case["d"]
        return {"bytes": e * (es + 2) + 2 * case["rows"] * _padded(case["d"]) // BLOCK + 2 * e, "flops": 6 * e}
    if case["op"] == "norm_step":
        p, c = case["n"] * case["h"] * case["w"], case["c"]
        e = p * c
        return {"bytes": 4 * e * es + 2 * (e + p * _padded(c) // BLOCK) + 24 * c + 16 * case["n"] * case["groups"],
                "flops": 28 * e}
    if case["op"] == "wgrad":
        t, d, o = case["rows"], case["d"], case["out"]
        return {"bytes": t * o * es + t * (d + _padded(d) // BLOCK) + 4 * o * (d + 1), "flops": 2 * t * d * o}
    t, d = case["rows"], case["d"]
    e = t * d
    gates = _gates(case)
    small = 4 * d * (3 + gates)
    if case["op"] == "block_fwd":
        return {"bytes": 4 * e * es + small + 16 * t, "flops": 16 * e}
    held = 2 * (e + t * _padded(d) // BLOCK) if case["kept"] else e * es
    return {"bytes": 8 * e * es + 2 * held + 2 * small + 32 * t, "flops": 50 * e}


def _gates(case):
    return 0 if case["gate"] == "none" else -(-case["rows"] // _per(case))


def _per(case):
    return case["rows"] if case["gate"] == "channel" else case["per"]


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def features(*shape):
        """Activations: each channel has its own spread and mean, a few stand far out."""
        x = normal(*shape)
        spread = torch.exp(0.5 * normal(shape[-1]))
        spread[torch.rand(shape[-1], generator=g, device="cuda") < 0.01] *= 12.0
        return x.mul_(spread).add_(0.3 * normal(shape[-1])).to(dt)

    s = {"case": dict(case)}
    if case["op"] == "ckpt":
        s["x"] = features(case["rows"], case["d"])
        s["kept"] = torch.empty(kept_bytes(case["rows"], case["d"]), dtype=torch.uint8, device="cuda")
        s["back"] = torch.empty((case["rows"], case["d"]), dtype=torch.bfloat16, device="cuda")
    elif case["op"] == "norm_step":
        shape = n, h, w, c = tuple(case[k] for k in ("n", "h", "w", "c"))
        s["x"], s["dy"] = features(*shape), normal(*shape).to(dt)
        s["gamma"], s["beta"] = 1.0 + 0.1 * normal(c), 0.1 * normal(c)
        s["y"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["stats"] = torch.empty((n, case["groups"], 2), device="cuda")
        s["dgamma"], s["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        s["kept"] = torch.empty(kept_bytes(n * h * w, c), dtype=torch.uint8, device="cuda")
    elif case["op"] == "wgrad":
        t, d, o = case["rows"], case["d"], case["out"]
        s["kept"] = keep(features(t, d))
        s["dy"] = normal(t, o).mul_(torch.exp(normal(t, 1))).mul_(1.0 / t).to(dt)
        s["dW"], s["db"] = torch.empty((o, d), device="cuda"), torch.empty(o, device="cuda")
    else:
        t, d, gates = case["rows"], case["d"], _gates(case)
        s["h"], s["u"] = features(t, d), features(t, d)
        s["pre"], s["post"] = 1.0 + 0.1 * normal(d), 1.0 + 0.1 * normal(d)
        s["shift"] = 0.1 * normal(d) if case["kind"] == "layer" else None
        s["gate"] = torch.tanh(normal(gates, d)) if gates else None
        s["keep"], s["scale"] = 1.0, 0.7
        s["h_out"], s["n"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
        s["stats"] = torch.empty((t, 4), device="cuda")
        if case["op"] == "block_step":
            s["dh_out"], s["dn"] = normal(t, d).to(dt), normal(t, d).to(dt)
            s["dh"], s["du"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
            for k in ("pre", "post", "shift", "gate"):
                s["d" + k] = torch.empty_like(s[k]) if s[k] is not None else None
            if case["kept"]:
                s["kept_h"], s["kept_u"] = (torch.empty(kept_bytes(t, d), dtype=torch.uint8, device="cuda")
                                            for _ in range(2))
    return s


# ---------------------------------------------------------------------------------------------------------------
# the form in which a tensor is kept: rows of whole numbers of 8 bits, padded with zeros to whole blocks, then the blocks'
# biased exponents.  A block's power of two is the least under which no value rounds beyond 127 (and at least 2^-126);
# halves round to even.
# ---------------------------------------------------------------------------------------------------------------
def kept_bytes(rows, d):
    return rows * _padded(d) + rows * _padded(d) // BLOCK


def keep(x):
    rows, d = x.shape
    dp = _padded(d)
    v = torch.zeros((rows, dp), device=x.device)
    v[:, :d] = x
    v = v.reshape(rows, dp // BLOCK, BLOCK)
    mantissa, exponent = torch.frexp(v.abs().amax(dim=2))
    k = torch.clamp(exponent - 7 + (mantissa >= 255 / 256), min=-126)
    k = torch.where(mantissa == 0, torch.full_like(k, -126), k)
    codes = torch.round(v * _power(-k)[:, :, None]).to(torch.int8)
    return torch.cat((codes.reshape(-1).view(torch.uint8), (k + 127).to(torch.uint8).reshape(-1)))


def _power(k):
    """2^k for whole k from -126 to 127."""
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def kept_values(kept, rows, d):
    dp = _padded(d)
    codes = kept[:rows * dp].view(torch.int8).reshape(rows, dp // BLOCK, BLOCK).float()
    k = kept[rows * dp:].reshape(rows, dp // BLOCK, 1).to(torch.int32) - 127
    return (codes * _power(k)).reshape(rows, dp)[:, :d]


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
        if c["op"] == "ckpt":
            s["q"] = dk.dk_ckpt8(c["rows"], c["d"], dt)
            s["q_back"] = dk.dk_ckpt8(c["rows"], c["d"], dk.DK_BF16)
        elif c["op"] == "norm_step":
            act = {"none": dk.DK_ACT_NONE, "silu": dk.DK_ACT_SILU}[c["act"]]
            s["q"] = dk.dk_norm(c["n"], c["h"], c["w"], c["c"], c["groups"], act, dt, EPS)
        elif c["op"] == "wgrad":
            s["q"] = dk.dk_wgrad8(c["rows"], c["d"], c["out"], dt)
        else:
            kind = dk.DK_BLOCK_RMS if c["kind"] == "rms" else dk.DK_BLOCK_LAYER
            s["q"] = dk.dk_block(c["rows"], c["d"], _per(c), kind, dt, EPS, s["keep"], s["scale"])
        if c["op"] != "ckpt":
            ctx.ensure_workspace(s["q"])
    q = s["q"]
    if c["op"] == "ckpt":
        dk.dk_ckpt8_store(ctx, q, s["x"], s["kept"])
        dk.dk_ckpt8_load(ctx, s["q_back"], s["kept"], s["back"])
        return {"back": s["back"]}
    if c["op"] == "norm_step":
        dk.dk_group_norm_fwd_ckpt8(ctx, q, s["x"], s["gamma"], s["beta"], s["y"], s["stats"], s["kept"])
        dk.dk_group_norm_bwd_ckpt8(ctx, q, s["dy"], s["kept"], s["gamma"], s["beta"], s["stats"], s["dx"], s["dgamma"],
                                   s["dbeta"])
        return {k: s[k] for k in ("y", "stats", "dx", "dgamma", "dbeta")}
    if c["op"] == "wgrad":
        dk.dk_linear_bwd_wgrad_ckpt8(ctx, q, s["dy"], s["kept"], 1.0, 0.0, s["dW"], s["db"])
        return {"dW": s["dW"], "db": s["db"]}
    dk.dk_block_norm_fwd(ctx, q, s["h"], s["u"], s["gate"], s["post"], s["pre"], s["shift"], s["h_out"], s["n"],
                         s["stats"], s.get("kept_h"), s.get("kept_u"))
    out = {k: s[k] for k in ("h_out", "n", "stats")}
    if c["op"] == "block_step":
        back = dk.dk_block_norm_bwd_ckpt8 if c["kept"] else dk.dk_block_norm_bwd
        h, u = (s["kept_h"], s["kept_u"]) if c["kept"] else (s["h"], s["u"])
        back(ctx, q, s["dh_out"], s["dn"], h, u, s["gate"], s["post"], s["pre"], s["stats"], s["dh"], s["du"], s["dgate"],
             s["dpost"], s["dpre"], s["dshift"])
        out.update({k: s[k] for k in ("dh", "du", "dpre", "dpost")})
        out.update({k: s[k] for k in ("dgate", "dshift") if s[k] is not None})
    return out


def _plain_ckpt(s):
    c = s["case"]
    return {"back": kept_values(keep(s["x"]), c["rows"], c["d"]).to(torch.bfloat16)}


def _plain_norm_step(s):
    c = s["case"]
    shape = (c["n"], c["h"] * c["w"], c["groups"], c["c"] // c["groups"])
    gamma, beta = s["gamma"].reshape(c["groups"], -1), s["beta"].reshape(c["groups"], -1)
    x = s["x"].float().reshape(shape)
    mean = x.mean(dim=(1, 3), keepdim=True)
    dev = x - mean
    rstd = 1.0 / torch.sqrt((dev * dev).mean(dim=(1, 3), keepdim=True) + EPS)
    z = dev * rstd * gamma + beta
    y = z if c["act"] == "none" else z / (1.0 + torch.exp(-z))
    kept = keep(s["x"].reshape(-1, c["c"]))
    # backward, from what was kept
    x = kept_values(kept, c["n"] * c["h"] * c["w"], c["c"]).reshape(shape)
    xhat = (x - mean) * rstd
    dz = s["dy"].float().reshape(shape)
    if c["act"] == "silu":
        z = xhat * gamma + beta
        sig = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * (sig * (1.0 + z * (1.0 - sig)))
    q = dz * gamma
    dx = rstd * (q - q.mean(dim=(1, 3), keepdim=True) - xhat * (q * xhat).mean(dim=(1, 3), keepdim=True))
    return {"y": y.reshape(s["x"].shape).to(s["x"].dtype), "stats": torch.stack((mean[:, 0, :, 0], rstd[:, 0, :, 0]), dim=-1),
            "dx": dx.reshape(s["x"].shape).to(s["x"].dtype), "dgamma": (dz * xhat).sum(dim=(0, 1)).reshape(-1),
            "dbeta": dz.sum(dim=(0, 1)).reshape(-1)}


def _plain_wgrad(s):
    c = s["case"]
    x, dy = kept_values(s["kept"], c["rows"], c["d"]), s["dy"].float()
    return {"dW": dy.t() @ x, "db": dy.sum(dim=0)}


def _normed(x, kind):
    mean = x.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    dev = x - mean
    rstd = 1.0 / torch.sqrt((dev * dev).mean(dim=1, keepdim=True) + EPS)
    return dev * rstd, mean, rstd


def _normed_back(q, xhat, rstd, kind):
    q = q - q.mean(dim=1, keepdim=True) - xhat * (q * xhat).mean(dim=1, keepdim=True) if kind == "layer" else \
        q - xhat * (q * xhat).mean(dim=1, keepdim=True)
    return rstd * q


def _gate_rows(s, dtype):
    """The gate of every row (None: 1)."""
    c = s["case"]
    if s["gate"] is None:
        return None
    return s["gate"].to(dtype)[torch.arange(c["rows"], device="cuda") // _per(c)]


def _sum_by_gate(s, v):
    """Sums over the rows that share a gate."""
    c = s["case"]
    gates, per = _gates(c), _per(c)
    if gates * per == c["rows"]:
        return v.reshape(gates, per, -1).sum(dim=1)
    whole = v[:(gates - 1) * per].reshape(gates - 1, per, v.shape[1]).sum(dim=1)
    return torch.cat((whole, v[(gates - 1) * per:].sum(dim=0, keepdim=True)))


def _plain_block(s):
    c, dt = s["case"], s["h"].dtype
    kind, gate = c["kind"], _gate_rows(s, torch.float32)
    h, u = s["h"].float(), s["u"].float()
    uhat, mean_u, rstd_u = _normed(u, kind)
    branch = uhat * s["post"]
    h_out = s["keep"] * h + s["scale"] * (branch if gate is None else gate * branch)
    hhat, mean_h, rstd_h = _normed(h_out, kind)
    n = hhat * s["pre"] if s["shift"] is None else hhat * s["pre"] + s["shift"]
    out = {"h_out": h_out.to(dt), "n": n.to(dt), "stats": torch.cat((mean_u, rstd_u, mean_h, rstd_h), dim=1)}
    if c["op"] == "block_fwd":
        return out
    if c["kept"]:
        h, u = (kept_values(keep(s[k]), c["rows"], c["d"]) for k in ("h", "u"))
        uhat = (u - mean_u) * rstd_u
        branch = uhat * s["post"]
        hhat = (s["keep"] * h + s["scale"] * (branch if gate is None else gate * branch) - mean_h) * rstd_h
    dn = s["dn"].float()
    D = s["dh_out"].float() + _normed_back(dn * s["pre"], hhat, rstd_h, kind)
    E = s["scale"] * D
    out["dh"] = (s["keep"] * D).to(dt)
    out["du"] = _normed_back((E if gate is None else E * gate) * s["post"], uhat, rstd_u, kind).to(dt)
    E = E * uhat
    out["dpre"], out["dpost"] = (dn * hhat).sum(dim=0), (E if gate is None else E * gate).sum(dim=0)
    if gate is not None:
        out["dgate"] = _sum_by_gate(s, E * s["post"])
    if s["shift"] is not None:
        out["dshift"] = dn.sum(dim=0)
    return out


_PLAIN = {"ckpt": _plain_ckpt, "norm_step": _plain_norm_step, "wgrad": _plain_wgrad, "block_fwd": _plain_block,
          "block_step": _plain_block}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _nearest(x):
    """What a kept tensor stands for: each value's nearest multiple of its block's power of two."""
    rows, d = x.shape
    v = torch.nn.functional.pad(x.to(torch.float64), (0, _padded(d) - d)).reshape(-1, BLOCK)
    top = v.abs().max(dim=1, keepdim=True).values
    at = torch.frexp(top).exponent.to(torch.int64) - 7           # top = m*2^(at + 7) with 1/2 <= m < 1
    step = ((at + 1023) << 52).view(torch.float64)
    step = torch.where(top / step >= 127.5, 2.0 * step, step).clamp(min=2.0 ** -126)
    return ((v / step).round() * step).reshape(rows, -1)[:, :d]


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "ckpt":
        return {"back": torch.cat([_nearest(part) for part in s["x"].split(1 << 18)])}
    if case["op"] == "norm_step":
        n, p, k, cg = case["n"], case["h"] * case["w"], case["groups"], case["c"] // case["groups"]
        gamma, beta = (s[t].to(f64).reshape(k, 1, cg) for t in ("gamma", "beta"))
        y, dx = (torch.empty(s["x"].shape, dtype=f64, device="cuda") for _ in range(2))
        stats = torch.empty((n, k, 2), dtype=f64, device="cuda")
        dgamma, dbeta = torch.zeros((k, cg), dtype=f64, device="cuda"), torch.zeros((k, cg), dtype=f64, device="cuda")
        for i in range(n):                        # one sample at a time, groups first: [k, p, cg]
            first = lambda t: t.to(f64).reshape(p, k, cg).transpose(0, 1)      # noqa: E731
            back = lambda t: t.transpose(0, 1).reshape(case["h"], case["w"], case["c"])      # noqa: E731
            x = first(s["x"][i])
            var, mean = torch.var_mean(x, dim=(1, 2), correction=0, keepdim=True)
            rstd = (var + EPS) ** -0.5
            z = (x - mean) * rstd * gamma + beta
            y[i] = back(z if case["act"] == "none" else z * torch.sigmoid(z))
            stats[i, :, 0], stats[i, :, 1] = mean[:, 0, 0], rstd[:, 0, 0]
            xhat = (first(_nearest(s["x"][i].reshape(p, -1))) - mean) * rstd
            z = xhat * gamma + beta
            sig = torch.sigmoid(z)
            d = first(s["dy"][i]) * (1.0 if case["act"] == "none" else sig + z * sig * torch.sigmoid(-z))
            dgamma += (d * xhat).sum(dim=1)
            dbeta += d.sum(dim=1)
            d = d * gamma
            a, b = d.sum(dim=(1, 2), keepdim=True) / (p * cg), (d * xhat).sum(dim=(1, 2), keepdim=True) / (p * cg)
            dx[i] = back((d - a - xhat * b) * rstd)
        return {"y": y, "stats": stats, "dx": dx, "dgamma": dgamma.reshape(-1), "dbeta": dbeta.reshape(-1)}
    if case["op"] == "wgrad":
        t, d, dp = case["rows"], case["d"], _padded(case["d"])
        dW = torch.zeros((case["out"], d), dtype=f64, device="cuda")
        db = torch.zeros(case["out"], dtype=f64, device="cuda")
        codes = s["kept"][:t * dp].view(torch.int8).reshape(t, dp)
        powers = torch.exp2(s["kept"][t * dp:].reshape(t, -1).to(f64) - 127.0)
        for a in range(0, t, 2048):
            x = codes[a:a + 2048].to(f64) * powers[a:a + 2048].repeat_interleave(BLOCK, dim=1)
            dy = s["dy"][a:a + 2048].to(f64)
            dW += torch.einsum("ro,rc->oc", dy, x[:, :d])
            db += dy.sum(dim=0)
        return {"dW": dW, "db": db}
    t, d, per, gates = case["rows"], case["d"], _per(case), _gates(case)
    layer = case["kind"] == "layer"
    post, pre = s["post"].to(f64), s["pre"].to(f64)
    shift = s["shift"].to(f64) if s["shift"] is not None else 0.0
    out = {k: torch.empty((t, d), dtype=f64, device="cuda") for k in ("h_out", "n", "dh", "du")}
    out["stats"] = torch.empty((t, 4), dtype=f64, device="cuda")
    sums = {k: torch.zeros(d, dtype=f64, device="cuda") for k in ("dpre", "dpost", "dshift")}
    dgate = torch.zeros((max(gates, 1), d), dtype=f64, device="cuda")

    def moments(v):
        mean = v.sum(dim=1, keepdim=True) / d if layer else torch.zeros((v.shape[0], 1), dtype=f64, device="cuda")
        return mean, (((v - mean) ** 2).sum(dim=1, keepdim=True) / d + EPS) ** -0.5

    def along(q, v, rstd):                         # gradient of (x - mean)*rstd, v the normalised values
        a = q.sum(dim=1, keepdim=True) / d if layer else 0.0
        return (q - a - v * ((q * v).sum(dim=1, keepdim=True) / d)) * rstd

    for a in range(0, t, 4096):
        at = slice(a, min(a + 4096, t))
        row = torch.arange(at.start, at.stop, device="cuda") // per
        gate = s["gate"].to(f64)[row] if gates else torch.ones((at.stop - at.start, 1), dtype=f64, device="cuda")
        h, u = s["h"][at].to(f64), s["u"][at].to(f64)
        mu, ru = moments(u)
        sum_ = s["keep"] * h + s["scale"] * gate * post * (u - mu) * ru
        mh, rh = moments(sum_)
        out["h_out"][at], out["n"][at] = sum_, (sum_ - mh) * rh * pre + shift
        out["stats"][at] = torch.cat((mu, ru, mh, rh), dim=1)
        if case["op"] == "block_fwd":
            continue
        if case["kept"]:
            h, u = _nearest(s["h"][at]), _nearest(s["u"][at])
        v = (u - mu) * ru
        w = (s["keep"] * h + s["scale"] * gate * post * v - mh) * rh
        dn = s["dn"][at].to(f64)
        D = s["dh_out"][at].to(f64) + along(dn * pre, w, rh)
        out["dh"][at] = s["keep"] * D
        out["du"][at] = along(s["scale"] * gate * post * D, v, ru)
        sums["dpre"] += (dn * w).sum(dim=0)
        sums["dshift"] += dn.sum(dim=0)
        sums["dpost"] += (s["scale"] * gate * D * v).sum(dim=0)
        dgate.index_add_(0, row, s["scale"] * post * D * v)
    if case["op"] == "block_fwd":
        return {k: out[k] for k in ("h_out", "n", "stats")}
    out.update(dpre=sums["dpre"], dpost=sums["dpost"])
    if gates:
        out["dgate"] = dgate
    if s["shift"] is not None:
        out["dshift"] = sums["dshift"]
    return out
