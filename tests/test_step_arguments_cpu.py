"""Argument checks of the training-step calls that need no GPU: the workspace sizes."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2207_00083_b200 import binding as dk


def size(q):
    n = ctypes.c_size_t()
    s = getattr(dk.lib(), f"{type(q).__name__}_workspace_bytes")(ctypes.byref(q), ctypes.byref(n))
    return s, n.value


def test_struct_layouts_match_header():
    assert ctypes.sizeof(dk.dk_norm) == 40 and dk.dk_norm.eps.offset == 32
    assert ctypes.sizeof(dk.dk_xent) == 24 and dk.dk_xent.dtype.offset == 16
    assert ctypes.sizeof(dk.dk_ortho) == 36


GOOD = [dk.dk_norm(4, 7, 7, 512, 32, 1, 0, 1e-5), dk.dk_norm(0, 1, 1, 1, 1, 0, 1, 0.0),
        dk.dk_xent(256, 4096, 1000, 0), dk.dk_xent(0, 1, 1, 1), dk.dk_xent(4096, 4096, 128000, 1),
        dk.dk_ortho(1, 4096, 25088, 0, 5, 3.4445, -4.775, 2.0315, 1e-7), dk.dk_ortho(3, 1, 1, 1, 0, 1.5, -0.5, 0.0, 0.0)]


@pytest.mark.parametrize("q", GOOD, ids=lambda q: type(q).__name__)
def test_accepted(q):
    s, n = size(q)
    assert s == 0 and n % 256 == 0


def test_workspace_holds_the_operands():
    # fp32: both terms of h and W, and of one piece of p
    s, n = size(dk.dk_xent(256, 4096, 1000, 0))
    assert n >= 4 * (256 * 4096 + 1000 * 4096 + 256 * 1000)
    # two generations of X, A and B
    s, n = size(dk.dk_ortho(2, 512, 4608, 0, 5, 3.4445, -4.775, 2.0315, 1e-7))
    assert n >= 4 * 2 * (2 * 512 * 4608 + 2 * 512 * 512)


SHAPE, INVALID = 2, 1
REFUSED = [
    (dk.dk_norm(1, 1, 1, 6, 4, 0, 0, 1e-5), SHAPE), (dk.dk_norm(1, 0, 1, 6, 2, 0, 0, 1e-5), SHAPE),
    (dk.dk_norm(-1, 1, 1, 6, 2, 0, 0, 1e-5), SHAPE), (dk.dk_norm(1, 1, 1, 20000, 2, 0, 0, 1e-5), SHAPE),
    (dk.dk_norm(1, 1, 1, 6, 0, 0, 0, 1e-5), SHAPE), (dk.dk_norm(1, 1, 1, 6, 2, 3, 0, 1e-5), INVALID),
    (dk.dk_norm(1, 1, 1, 6, 2, 0, 2, 1e-5), INVALID), (dk.dk_norm(1, 1, 1, 6, 2, 0, 0, -1.0), INVALID),
    (dk.dk_norm(1, 1, 1, 6, 2, 0, 0, float("nan")), INVALID), (dk.dk_norm(1, 65536, 65536, 1, 1, 0, 0, 1e-5), SHAPE),
    (dk.dk_xent(-1, 8, 8, 0), SHAPE), (dk.dk_xent(8, 0, 8, 0), SHAPE), (dk.dk_xent(8, 8, 0, 0), SHAPE),
    (dk.dk_xent(8, 8, 8, 5), INVALID), (dk.dk_xent(1 << 30, 8, 8, 0), SHAPE),
    (dk.dk_ortho(0, 8, 8, 0, 5, 1.5, -0.5, 0.0, 0.0), SHAPE), (dk.dk_ortho(1, 0, 8, 0, 5, 1.5, -0.5, 0.0, 0.0), SHAPE),
    (dk.dk_ortho(1, 8, 70000, 0, 5, 1.5, -0.5, 0.0, 0.0), SHAPE), (dk.dk_ortho(1, 8, 8, 0, 33, 1.5, -0.5, 0.0, 0.0), SHAPE),
    (dk.dk_ortho(1, 8, 8, 3, 5, 1.5, -0.5, 0.0, 0.0), INVALID), (dk.dk_ortho(1, 8, 8, 0, 5, 40.0, -0.5, 0.0, 0.0), INVALID),
    (dk.dk_ortho(1, 8, 8, 0, 5, float("nan"), -0.5, 0.0, 0.0), INVALID),
    (dk.dk_ortho(1, 8, 8, 0, 5, 1.5, -0.5, 0.0, -1.0), INVALID),
]


@pytest.mark.parametrize("q,status", REFUSED)
def test_refused(q, status):
    assert size(q)[0] == status


def test_null_arguments():
    L = dk.lib()
    n = ctypes.c_size_t()
    for t in ("norm", "xent", "ortho"):
        f = getattr(L, f"dk_{t}_workspace_bytes")
        assert f(None, ctypes.byref(n)) == INVALID
    q = dk.dk_norm(1, 1, 1, 6, 2, 0, 0, 1e-5)
    assert L.dk_norm_workspace_bytes(ctypes.byref(q), None) == INVALID
    assert L.dk_group_norm_fwd(None, ctypes.byref(q), None, None, None, None, None, None) == INVALID
    x = dk.dk_xent(8, 8, 8, 0)
    assert L.dk_linear_xent_fwd(None, ctypes.byref(x), None, None, None, None, None, None) == INVALID
    o = dk.dk_ortho(1, 8, 8, 0, 5, 1.5, -0.5, 0.0, 0.0)
    assert L.dk_orthogonalize(None, ctypes.byref(o), None, 1.0, 0.0, None, None) == INVALID


@pytest.mark.parametrize("h,w,c", [(46340, 46340, 1), (1, 2 ** 31 - 4096, 1), (1, 2 ** 31 - 4096, 8), (2, 2 ** 30 - 2048, 3)])
def test_images_of_almost_two_to_the_31_pixels(h, w, c):
    """The number of slabs is formed in 64 bits: the workspace is some slabs' sums, far less than the tensor."""
    s, n = size(dk.dk_norm(1, h, w, c, 1, 0, 1, 1e-5))
    assert s == 0 and 0 < n < 64 << 20


@pytest.mark.parametrize("h,w", [(1, 2 ** 31 - 4095), (1, 2 ** 31 - 1), (46341, 46341)])
def test_images_past_the_limit_are_refused(h, w):
    assert size(dk.dk_norm(1, h, w, 1, 1, 0, 1, 1e-5))[0] == SHAPE


class Elsewhere:
    """What the binding asks of a tensor, on a device of choice."""

    def __init__(self, device, numel, dtype):
        self.device_index, self.n, self.dtype, self.is_cuda = device, numel, dtype, device >= 0

    def get_device(self):
        return self.device_index

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


NORM, XENT, ORTHO = dk.dk_norm(2, 3, 3, 8, 2, 1, 0, 1e-5), dk.dk_xent(4, 8, 16, 0), dk.dk_ortho(1, 8, 8, 0, 5, 1.5, -0.5, 0.0, 0.0)
CONV = dk.dk_problem(dk.DK_FC, dk.DK_NHWC, 8, 8, 1, 1, 1, 1, 1, 0, 4, 1, 0, 0.0)
F, I64, I32 = torch.float32, torch.int64, torch.int32
COEF = np.zeros((1, 6, 5), np.float32)
CALLS = {
    "dk_group_norm_fwd": (lambda f, c, t: f(c, NORM, *t), [(144, F), (8, F), (8, F), (144, F), (8, F)]),
    "dk_group_norm_bwd": (lambda f, c, t: f(c, NORM, *t), [(144, F), (144, F), (8, F), (8, F), (8, F), (144, F), (8, F), (8, F)]),
    "dk_linear_xent_fwd": (lambda f, c, t: f(c, XENT, *t), [(32, F), (128, F), (4, I64), (4, F), (4, F)]),
    "dk_linear_xent_bwd": (lambda f, c, t: f(c, XENT, *t[:5], 1.0, *t[5:]),
                           [(32, F), (128, F), (4, I64), (4, F), (4, F), (32, F), (128, F)]),
    "dk_orthogonalize": (lambda f, c, t: f(c, ORTHO, t[0], 1.0, 0.0, t[1]), [(64, F), (64, F)]),
    "dk_encode": (lambda f, c, t: f(c, CONV, t[0], t[1], COEF, t[2]), [(32, F), (8, F), (48, F)]),
    "dk_linear_bwd_dgrad": (lambda f, c, t: f(c, CONV, *t), [(64, F), (32, F), (32, F)]),
    "dk_relu_pool_fwd": (lambda f, c, t: f(c, t[0], 4, 1, 1, 8, False, t[1]), [(32, F), (32, F)]),
    "dk_field_quantize": (lambda f, c, t: f(c, t[0], 8, 2 ** 25 - 39, t[1]), [(32, F), (32, I32)]),
}


@pytest.mark.parametrize("device,other", [(0, 1), (1, 0), (0, -1)])
@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(name, device, other, monkeypatch):
    """Each argument in turn lies on another device than the context (or on the host): refused before the library sees a
    pointer; with all of them in place the library is reached (and refuses the missing context)."""
    monkeypatch.setattr(dk, "_raw_stream", lambda d: 0)
    call, sizes = CALLS[name]
    ctx = SimpleNamespace(handle=None, device=device)
    for wrong in range(len(sizes)):
        tensors = [Elsewhere(other if i == wrong else device, *s) for i, s in enumerate(sizes)]
        with pytest.raises(ValueError):
            call(getattr(dk, name), ctx, tensors)
    with pytest.raises(dk.DkError) as e:
        call(getattr(dk, name), ctx, [Elsewhere(device, *s) for s in sizes])
    assert e.value.status == INVALID


@pytest.mark.parametrize("rows,d,vocab,dtype", [(1, 2048, 128000, 0), (1, 2048, 128000, 1), (8, 1024, 50257, 0), (64, 512, 1000, 0),
                                                (2047, 1024, 50257, 1), (300, 100, 5001, 1), (0, 1, 1, 0), (1, 30000, 40, 0)])
def test_scoring_needs_no_more_than_both_directions(rows, d, vocab, dtype):
    q, n = dk.dk_xent(rows, d, vocab, dtype), ctypes.c_size_t()
    assert dk.lib().dk_xent_fwd_workspace_bytes(ctypes.byref(q), ctypes.byref(n)) == 0
    es = 4 if dtype == 0 else 2
    assert n.value % 256 == 0 and n.value <= size(q)[1]
    if rows <= 8 and 1 <= rows and d <= 2048 and dtype == 0 or rows == 1 and d <= 8192:
        assert n.value < 64 << 10                               # dot products: nothing is laid out anew
    if dtype == 1 and d % 8 == 0:
        assert n.value < (64 << 20) + 8 * rows * vocab // 128 + 16 * rows      # operands are read in place
    assert n.value < (64 << 20) + 2 * es * (rows + vocab) * (d + 8) + 8 * rows * (vocab // 128 + 1)


def test_scoring_workspace_refusals():
    n = ctypes.c_size_t()
    assert dk.lib().dk_xent_fwd_workspace_bytes(None, ctypes.byref(n)) == INVALID
    assert dk.lib().dk_xent_fwd_workspace_bytes(ctypes.byref(dk.dk_xent(8, 0, 8, 0)), ctypes.byref(n)) == SHAPE
