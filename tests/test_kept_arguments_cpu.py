"""Argument checks of the checkpoint and block calls that need no GPU.  A context of zeros stands in where a refusal comes
before the context is looked into."""
import ctypes
from types import SimpleNamespace

import pytest
import torch

import kept
from paper_2207_00083_b200 import binding as dk

OK, INVALID, SHAPE, WORKSPACE = 0, 1, 2, 4
NAN, INF = float("nan"), float("inf")
SIZES = {"dk_ckpt8": "dk_ckpt8_bytes", "dk_wgrad8": "dk_wgrad8_workspace_bytes", "dk_block": "dk_block_workspace_bytes"}


def size(q):
    n = ctypes.c_size_t()
    return getattr(dk.lib(), SIZES[type(q).__name__])(ctypes.byref(q), ctypes.byref(n)), n.value


def test_struct_layouts_match_header():
    assert ctypes.sizeof(dk.dk_ckpt8) == 16 and ctypes.sizeof(dk.dk_wgrad8) == 24 and dk.dk_wgrad8.dtype.offset == 16
    assert ctypes.sizeof(dk.dk_block) == 48 and dk.dk_block.rows_per_gate.offset == 16 and dk.dk_block.eps.offset == 32


@pytest.mark.parametrize("rows,d", [(0, 1), (1, 1), (3, 32), (3, 33), (1 << 25, 64), (7, 1 << 20)])
def test_checkpoint_size(rows, d):
    for t in (dk.DK_F32, dk.DK_BF16):
        assert size(dk.dk_ckpt8(rows, d, t)) == (OK, kept.size(rows, d))


def block(rows=4, d=8, per=1, kind=0, dtype=0, eps=1e-5, keep=1.0, scale=1.0):
    return dk.dk_block(rows, d, per, kind, dtype, eps, keep, scale)


@pytest.mark.parametrize("q", [dk.dk_wgrad8(0, 1, 1, 0), dk.dk_wgrad8(64, 512, 1000, 0), dk.dk_wgrad8(5, 1 << 20, 3, 1),
                               dk.dk_wgrad8(5, 3, (1 << 20) - 1, 0), block(0), block(1, 1), block(70000, 16384, 1, 1, 1),
                               block(1 << 20, 64, 1 << 40)], ids=lambda q: type(q).__name__)
def test_accepted(q):
    s, n = size(q)
    assert s == OK and n % 256 == 0


def test_workspaces_hold_what_is_laid_out():
    assert size(dk.dk_wgrad8(1000, 512, 777, 0))[1] >= 1000 * (512 * 2 + 777 * 4)
    assert size(dk.dk_wgrad8(1000, 512, 776, 1))[1] >= 1000 * 512 * 2
    # parts of the sums over rows, not copies of the rows
    assert size(block(100000, 1024, 1, 1, 0))[1] < 100000 * 1024


REFUSED = [(dk.dk_ckpt8(-1, 8, 0), SHAPE), (dk.dk_ckpt8(1, 0, 0), SHAPE), (dk.dk_ckpt8(1, (1 << 20) + 1, 0), SHAPE),
           (dk.dk_ckpt8(1 << 40, 8, 0), SHAPE), (dk.dk_ckpt8(1, 8, 2), INVALID), (dk.dk_wgrad8(-1, 8, 8, 0), SHAPE),
           (dk.dk_wgrad8(8, 0, 8, 0), SHAPE), (dk.dk_wgrad8(8, 8, 0, 0), SHAPE), (dk.dk_wgrad8((1 << 24) + 1, 8, 8, 0), SHAPE),
           (dk.dk_wgrad8(8, 8, 8, 7), INVALID), (block(-1), SHAPE), (block(4, 0), SHAPE), (block(4, 16385), SHAPE),
           (block(4, 8, 0), SHAPE), (block(4, 8, -3), SHAPE), (block((1 << 30) + 1, 8), SHAPE), (block(kind=2), INVALID),
           (block(dtype=2), INVALID), (block(eps=-1.0), INVALID), (block(eps=NAN), INVALID), (block(keep=INF), INVALID),
           (block(scale=NAN), INVALID)]


@pytest.mark.parametrize("q,status", REFUSED, ids=lambda v: type(v).__name__)
def test_refused_sizes(q, status):
    assert size(q)[0] == status
    assert getattr(dk.lib(), SIZES[type(q).__name__])(ctypes.byref(q), None) == INVALID


FAKE = (ctypes.c_char * 65536)()
P = 1 << 20                            # "tensors", far apart: nothing is read before a refusal


def at(i):
    return P + 4096 * i


def fwd(q, **change):
    a = dict(h=at(1), u=at(2), gate=at(3), post=at(4), pre=at(5), shift=at(6), h_out=at(7), n=at(8), stats=at(9), kh=at(10),
             ku=at(11), ctx=ctypes.addressof(FAKE))
    a.update(change)
    return dk.lib().dk_block_norm_fwd(a["ctx"], ctypes.byref(q), *[a[k] for k in ("h", "u", "gate", "post", "pre", "shift", "h_out",
                                                                                 "n", "stats", "kh", "ku")], None)


def bwd(q, name="dk_block_norm_bwd", **change):
    order = ("dh_out", "dn", "h", "u", "gate", "post", "pre", "stats", "dh", "du", "dgate", "dpost", "dpre", "dshift")
    a = {k: at(i + 1) for i, k in enumerate(order)}
    a["ctx"] = ctypes.addressof(FAKE)
    a.update(change)
    return getattr(dk.lib(), name)(a["ctx"], ctypes.byref(q), *[a[k] for k in order], None)


@pytest.mark.parametrize("change", [dict(ctx=None), dict(h=None), dict(u=None), dict(post=None), dict(h_out=None), dict(n=None),
                                    dict(pre=None), dict(h=at(1) + 4), dict(gate=at(3) + 8), dict(kh=at(10) + 1), dict(n=at(1)),
                                    dict(n=at(2)), dict(n=at(7)), dict(h_out=at(2)), dict(ku=at(10)),
                                    dict(u=None, post=None, h_out=None), dict(u=None, post=None, h_out=None, gate=None),
                                    dict(n=None, pre=None),
                                    dict(u=None, post=None, h_out=None, gate=None, ku=None, n=None, pre=None, shift=None)])
def test_refused_forward(change):
    assert fwd(block(), **change) == INVALID


@pytest.mark.parametrize("name", ["dk_block_norm_bwd", "dk_block_norm_bwd_ckpt8"])
@pytest.mark.parametrize("change", [dict(ctx=None), dict(h=None), dict(u=None), dict(du=None), dict(post=None), dict(dpost=None),
                                    dict(gate=None), dict(dgate=None), dict(dn=None), dict(pre=None), dict(dpre=None), dict(stats=None),
                                    dict(dh=None), dict(dn=None, dh_out=None), dict(dn=None, pre=None, dpre=None),
                                    dict(dn=None, pre=None, dpre=None, dshift=None, dh_out=None), dict(dh=at(2)), dict(dh=at(3)),
                                    dict(dh=at(4)), dict(du=at(9)), dict(du=at(1)), dict(du=at(2)), dict(du=at(4)),
                                    dict(dh_out=at(1) + 2), dict(dpre=at(13) + 4)])
def test_refused_backward(name, change):
    assert bwd(block(), name, **change) == INVALID


def test_refused_others():
    L, ctx = dk.lib(), ctypes.addressof(FAKE)
    k, w, n = dk.dk_ckpt8(4, 8, 0), dk.dk_wgrad8(4, 8, 8, 0), dk.dk_norm(2, 3, 3, 8, 2, 1, 0, 1e-5)
    for call in (L.dk_ckpt8_store, L.dk_ckpt8_load):
        for a in ((None, at(1), at(2)), (ctx, None, at(2)), (ctx, at(1), None), (ctx, at(1) + 4, at(2)), (ctx, at(1), at(2) + 8)):
            assert call(a[0], ctypes.byref(k), a[1], a[2], None) == INVALID
    good = [ctx, at(1), at(2), 1.0, 0.0, at(3), at(4)]
    for i, v in ((0, None), (1, None), (2, None), (5, None), (3, NAN), (3, INF), (4, NAN), (1, at(1) + 2), (6, at(4) + 4)):
        a = list(good)
        a[i] = v
        assert L.dk_linear_bwd_wgrad_ckpt8(a[0], ctypes.byref(w), a[1], a[2], a[3], a[4], a[5], a[6], None) == INVALID
    for i in range(1, 7):
        a = [ctx] + [at(j) for j in range(1, 7)]
        a[i] = None
        assert L.dk_group_norm_fwd_ckpt8(a[0], ctypes.byref(n), *a[1:], None) == INVALID
        a[i] = at(i) + 4
        assert L.dk_group_norm_fwd_ckpt8(a[0], ctypes.byref(n), *a[1:], None) == INVALID
    for i in range(1, 9):
        a = [ctx] + [at(j) for j in range(1, 9)]
        a[i] = None
        assert L.dk_group_norm_bwd_ckpt8(a[0], ctypes.byref(n), *a[1:], None) == INVALID


class Elsewhere:
    """What the binding asks of a tensor, on a device of choice."""

    def __init__(self, device, numel, dtype):
        self.device_index, self.n, self.dtype = device, numel, dtype

    def get_device(self):
        return self.device_index

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


F, U8 = torch.float32, torch.uint8
KEPT, WG, NORM, BLOCK = dk.dk_ckpt8(4, 8, 0), dk.dk_wgrad8(4, 8, 16, 0), dk.dk_norm(2, 3, 3, 8, 2, 1, 0, 1e-5), block(4, 8, 3)
K = (4 * 33, U8)
CALLS = {
    "dk_ckpt8_store": (lambda f, c, t: f(c, KEPT, *t), [(32, F), K]),
    "dk_ckpt8_load": (lambda f, c, t: f(c, KEPT, *t), [K, (32, F)]),
    "dk_group_norm_fwd_ckpt8": (lambda f, c, t: f(c, NORM, *t), [(144, F), (8, F), (8, F), (144, F), (8, F), (18 * 33, U8)]),
    "dk_group_norm_bwd_ckpt8": (lambda f, c, t: f(c, NORM, *t),
                                [(144, F), (18 * 33, U8), (8, F), (8, F), (8, F), (144, F), (8, F), (8, F)]),
    "dk_linear_bwd_wgrad_ckpt8": (lambda f, c, t: f(c, WG, t[0], t[1], 1.0, 0.0, t[2], t[3]), [(64, F), K, (128, F), (16, F)]),
    "dk_block_norm_fwd": (lambda f, c, t: f(c, BLOCK, *t), [(32, F), (32, F), (16, F), (8, F), (8, F), (8, F), (32, F), (32, F),
                                                            (16, F), K, K]),
    "dk_block_norm_bwd": (lambda f, c, t: f(c, BLOCK, *t), [(32, F)] * 4 + [(16, F), (8, F), (8, F), (16, F), (32, F), (32, F), (16, F),
                                                                            (8, F), (8, F), (8, F)]),
    "dk_block_norm_bwd_ckpt8": (lambda f, c, t: f(c, BLOCK, *t), [(32, F)] * 2 + [K, K, (16, F), (8, F), (8, F), (16, F), (32, F),
                                                                                  (32, F), (16, F), (8, F), (8, F), (8, F)]),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_that_do_not_fit_are_refused(name, monkeypatch):
    """Each argument in turn on another device, of another size or of another type: refused before the library sees a
    pointer; with all of them in place the library is reached (and refuses the missing context)."""
    monkeypatch.setattr(dk, "_raw_stream", lambda d: 0)
    call, sizes = CALLS[name]
    ctx = SimpleNamespace(handle=None, device=0)
    for wrong in range(len(sizes)):
        n, t = sizes[wrong]
        for bad in (Elsewhere(1, n, t), Elsewhere(-1, n, t), Elsewhere(0, n + 1, t), Elsewhere(0, n, torch.float64)):
            tensors = [bad if i == wrong else Elsewhere(0, *s) for i, s in enumerate(sizes)]
            with pytest.raises(ValueError):
                call(getattr(dk, name), ctx, tensors)
    with pytest.raises(dk.DkError) as e:
        call(getattr(dk, name), ctx, [Elsewhere(0, *s) for s in sizes])
    assert e.value.status == INVALID
