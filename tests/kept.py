"""The 8-bit form of a checkpoint in 64 bits, for the tests: found by trying powers of two, not by the formula on bits."""
import torch

BLOCK = 32


def padded(d):
    return -(-d // BLOCK) * BLOCK


def size(rows, d):
    return rows * padded(d) + rows * padded(d) // BLOCK


def parts(kept, rows, d):
    """Codes [rows][padded] and exponent bytes [rows][blocks] of a checkpoint."""
    n = rows * padded(d)
    return kept[:n].view(torch.int8).reshape(rows, padded(d)), kept[n:].reshape(rows, padded(d) // BLOCK)


def encode(x):
    """Codes and exponent bytes of x[rows][d], float64 arithmetic throughout."""
    rows, d = x.shape
    v = torch.zeros((rows, padded(d)), dtype=torch.float64, device=x.device)
    v[:, :d] = x.double()
    v = v.reshape(rows, -1, BLOCK)
    top = v.abs().amax(dim=2)
    bad = ~torch.isfinite(v).all(dim=2)
    v, top = torch.where(bad[:, :, None], torch.zeros_like(v), v), torch.where(bad, torch.zeros_like(top), top)
    b = torch.ones(top.shape, dtype=torch.int64, device=x.device)
    for bit in (128, 64, 32, 16, 8, 4, 2, 1):                # the least b at which the largest value fits
        trial = (b + bit - 1).clamp(max=254)
        b = torch.where(torch.round(top * power(127 - trial)) > 127, b + bit, b)
    b = b.clamp(max=248)
    q = torch.round(v * power(127 - b)[:, :, None]).clamp(-127, 127)
    b = torch.where(bad, torch.full_like(b, 255), b)
    return q.reshape(rows, -1).to(torch.int8), b.to(torch.uint8)


def power(k):
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def values(codes, exps, d):
    """What the checkpoint stands for, in 64 bits."""
    rows = codes.shape[0]
    v = codes.double().reshape(rows, -1, BLOCK) * power(exps.to(torch.int64) - 127)[:, :, None]
    v = torch.where((exps == 255)[:, :, None], torch.full_like(v, float("nan")), v)
    return v.reshape(rows, -1)[:, :d]


def decode(kept, rows, d):
    return values(*parts(kept, rows, d), d)


def pack(codes, exps):
    return torch.cat((codes.reshape(-1).view(torch.uint8), exps.reshape(-1)))
