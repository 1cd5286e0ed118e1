"""Workspaces of the dense layers' C ABI, without a GPU: what may not overlap
them, and how large they are.  The checks and the size query come before any
HIP call (the device pointers are made up and never followed)."""
import ctypes

import pytest
import torch

from paper_1512_06473_amd import _lib, quantize_net

ALIAS, WORKSPACE = 7, 8
F32, BF16, F16 = 0, 1, 2


def at(n):
    return n << 36  # arrays 64 GiB apart


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


LINEAR = dict(dtype=BF16, x=at(1), ldx=64, N=40, Cs=64, w=at(2), Ct=32, bias=at(3), act=4, residual=at(4), ldr=32,
              pre=at(5), y=at(6), ldy=32)
GRAD = dict(dtype=BF16, dy=at(1), lddy=32, x=at(2), ldx=64, N=40, Cs=64, w=at(3), Ct=32, pre=at(4), act=2, dx=at(5),
            dw=at(6), dbias=at(7))
GATED = dict(dtype=F16, x=at(1), ldx=64, N=40, Cs=64, w=at(2), Ct=32, bias=at(3), act=4, pre=at(5), y=at(6), ldy=32)
XENT = dict(dtype=F32, x=at(1), ldx=64, N=40, Cs=64, w=at(2), Ct=32, bias=at(3), labels=at(4), loss=at(5), lse=at(6))
XGRAD = dict(dtype=F32, dloss=at(8), lse=at(6), x=at(1), ldx=64, N=40, Cs=64, w=at(2), Ct=32, bias=at(3),
             labels=at(4), dx=at(9), dw=at(10), dbias=at(11))
CALLS = {"qcnn_linear_forward": LINEAR, "qcnn_linear_backward": GRAD, "qcnn_gated_forward": GATED,
         "qcnn_gated_backward": GRAD, "qcnn_linear_xent_forward": XENT, "qcnn_linear_xent_backward": XGRAD}


@pytest.mark.parametrize("entry,name", [(e, k) for e, args in CALLS.items() for k, v in args.items() if v >= at(1)])
def test_a_workspace_overlaps_no_argument(L, entry, name):
    """It is written like an output: no input, not even its last byte, may lie in it."""
    f, args = getattr(L, entry), CALLS[entry]
    size = ctypes.c_size_t(1 << 20)
    assert f(*args.values(), args[name], ctypes.byref(size), None) == ALIAS          # on it
    assert f(*args.values(), args[name] - (1 << 19), ctypes.byref(size), None) == ALIAS  # reaching into it
    size = ctypes.c_size_t(2 ** 64 - 1)                                               # as long as can be said
    assert f(*args.values(), args[name] - (1 << 19), ctypes.byref(size), None) == ALIAS
    # right in front of it: past the check, and refused as too small before anything is launched
    size = ctypes.c_size_t(256)
    args = dict(args, Cs=65, ldx=65, N=200)  # larger than the caller's 256 bytes
    assert f(*args.values(), args[name] - 256, ctypes.byref(size), None) == WORKSPACE


def need(L, entry, args):
    n = ctypes.c_size_t(0)
    assert getattr(L, entry)(*args.values(), None, ctypes.byref(n), None) == 0
    return n.value


@pytest.mark.parametrize("entry,halves", [("qcnn_linear_backward", 1), ("qcnn_gated_backward", 2)])
@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("Cs", [4096, 4095])
def test_nothing_is_reserved_for_what_is_not_read(L, entry, halves, act, Cs):
    """4095 columns of a 16-bit type are copied to rows of 4096: of x for dw
    only, of w for dx only.  dbias alone needs its sums, no dz."""
    N, rows = 4096, halves * 4096
    full = dict(GRAD, N=N, Cs=Cs, ldx=Cs, Ct=4096, lddy=4096, act=act)
    full = {k: v << 2 if v >= at(1) else v for k, v in full.items()}
    whole = need(L, entry, full)
    dbias = need(L, entry, dict(full, dx=None, dw=None, x=None, w=None))
    assert dbias <= 512 * rows * 4 + 256
    copies = (2 * 4096 * N, 2 * 4096 * rows) if Cs % 2 else (0, 0)
    assert need(L, entry, dict(full, dx=None, w=None)) <= whole - copies[1]
    assert need(L, entry, dict(full, dw=None, x=None)) <= whole - copies[0]


def test_responses_take_no_product_that_nobody_reads(monkeypatch):
    """One product per layer without a bias; two with one (the response has
    none), but for the last layer, whose output no layer reads."""
    calls = []

    def linear(x, w, bias=None, act="none", residual=None, out=None, pre=None):
        z = x @ w.t()
        if pre is not None:
            pre.copy_(z if bias is None else z + bias)
        calls.append((tuple(w.shape), act))
        z = z if bias is None else z + bias
        return torch.relu(z) if act == "relu" else z

    monkeypatch.setattr(quantize_net.api, "linear_forward", linear)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 2, 4, generator=g)
    for biased in (True, False):
        calls.clear()
        specs = [{"kind": "fc", "W": torch.randn(ct, cs, generator=g), "relu": True,
                  "bias": torch.randn(ct, generator=g) if biased else None} for cs, ct in ((8, 6), (6, 7), (7, 3))]
        got, h = quantize_net.fc_responses(x, specs), x.reshape(5, 8)
        for t, s in zip(got, specs):
            z = h @ s["W"].t()
            assert torch.equal(t, z)
            h = torch.relu(z + s["bias"] if biased else z)
        assert len(calls) == (5 if biased else 3)
    assert quantize_net.fc_responses(x, []) == []
