"""Refusals and workspace sizes of the dense layers' C ABI, without a GPU:
validation and the size query come before any HIP call (the device pointers
are made up and never followed)."""
import ctypes

import pytest
import torch

from paper_1512_06473_amd import _lib, api

NULL, SHAPE, UNSUP, ALIAS, WORKSPACE = 1, 2, 6, 7, 8
F32, BF16, F16 = 0, 1, 2


def at(n):
    return n << 32  # arrays 4 GiB apart


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def size(entry, args):
    n = ctypes.c_size_t(12345)
    rc = entry(*args, None, ctypes.byref(n), None)
    return rc, n.value


LINEAR = dict(dtype=BF16, x=at(1), ldx=64, N=8, Cs=64, w=at(2), Ct=32, bias=at(3), act=4, res=at(4), ldr=32,
              pre=at(5), y=at(6), ldy=32)
GRAD = dict(dtype=BF16, dy=at(1), lddy=32, x=at(2), ldx=64, N=8, Cs=64, w=at(3), Ct=32, pre=at(4), act=2, dx=at(5),
            dw=at(6), dbias=at(7))
GATED = dict(dtype=F16, x=at(1), ldx=64, N=8, Cs=64, w=at(2), Ct=32, bias=at(3), act=4, pre=at(5), y=at(6), ldy=32)
XENT = dict(dtype=F32, x=at(1), ldx=64, N=8, Cs=64, w=at(2), Ct=32, bias=at(3), labels=at(4), loss=at(5), lse=at(6))
XGRAD = dict(dtype=F32, dloss=at(8), lse=at(6), x=at(1), ldx=64, N=8, Cs=64, w=at(2), Ct=32, bias=at(3),
             labels=at(4), dx=at(9), dw=at(10), dbias=at(11))
CALLS = {"qcnn_linear_forward": LINEAR, "qcnn_linear_backward": GRAD, "qcnn_gated_forward": GATED,
         "qcnn_gated_backward": GRAD, "qcnn_linear_xent_forward": XENT, "qcnn_linear_xent_backward": XGRAD}
HUGE = 1 << 21

COMMON = [(dict(N=0), SHAPE), (dict(N=-1), SHAPE), (dict(Cs=0), SHAPE), (dict(Ct=0), SHAPE), (dict(ldx=63), SHAPE),
          (dict(dtype=3), UNSUP), (dict(dtype=-1), UNSUP), (dict(N=HUGE + 1), UNSUP), (dict(ldx=HUGE), UNSUP),
          (dict(x=None), NULL), (dict(w=None), NULL), (dict(x=at(1) + 1), UNSUP), (dict(w=at(2) + 1), UNSUP)]
CASES = [("qcnn_linear_forward", kw, want) for kw, want in COMMON + [
    (dict(y=None), NULL), (dict(act=5), UNSUP), (dict(act=-1), UNSUP), (dict(ldy=31), SHAPE), (dict(ldr=31), SHAPE),
    (dict(y=at(1)), ALIAS), (dict(y=at(1) + 16 * 63), ALIAS), (dict(y=at(4)), ALIAS), (dict(pre=at(6)), ALIAS),
    (dict(pre=at(2)), ALIAS), (dict(y=at(3)), ALIAS), (dict(y=at(6) + 1), UNSUP),
    (dict(N=HUGE, Ct=1 << 20, ldy=1 << 20, ldr=1 << 20), UNSUP),                  # tiles
]]
CASES += [(e, kw, want) for e in ("qcnn_linear_backward", "qcnn_gated_backward") for kw, want in COMMON + [
    (dict(dy=None), NULL), (dict(pre=None), NULL), (dict(dx=None, dw=None, dbias=None), NULL), (dict(lddy=31), SHAPE),
    (dict(dx=at(1)), ALIAS), (dict(dw=at(3)), ALIAS), (dict(dw=at(5)), ALIAS), (dict(dbias=at(4)), ALIAS)]]
CASES += [("qcnn_gated_forward", kw, want) for kw, want in COMMON + [
    (dict(y=None), NULL), (dict(act=7), UNSUP), (dict(ldy=31), SHAPE), (dict(y=at(1)), ALIAS), (dict(pre=at(6)), ALIAS),
    (dict(Ct=(1 << 19) + 1, ldy=1 << 20), UNSUP)]]                                  # 2 C_t rows
CASES += [("qcnn_linear_xent_forward", kw, want) for kw, want in COMMON + [
    (dict(labels=None), NULL), (dict(loss=None), NULL), (dict(lse=None), NULL), (dict(labels=at(4) + 4), UNSUP),
    (dict(loss=at(5) + 2), UNSUP), (dict(loss=at(6)), ALIAS), (dict(lse=at(4)), ALIAS)]]
CASES += [("qcnn_linear_xent_backward", kw, want) for kw, want in COMMON + [
    (dict(labels=None), NULL), (dict(dloss=None), NULL), (dict(lse=None), NULL),
    (dict(dx=None, dw=None, dbias=None), NULL), (dict(dx=at(2)), ALIAS), (dict(dw=at(6)), ALIAS),
    (dict(dbias=at(8)), ALIAS), (dict(dw=at(9)), ALIAS)]]


@pytest.mark.parametrize("entry,kw,want", CASES)
def test_rejects(L, entry, kw, want):
    if entry.endswith("_backward") and "xent" not in entry:  # other places of x and w there
        kw = {k: (at(2) + 1 if k == "x" else at(3) + 1) if k in "xw" and v is not None else v for k, v in kw.items()}
    args = dict(CALLS[entry], **kw)
    assert getattr(L, entry)(*args.values(), None, None, None) == want
    rc, n = size(getattr(L, entry), args.values())
    assert rc == want and n == 12345  # a refused query writes nothing


@pytest.mark.parametrize("entry", list(CALLS))
def test_size_query_and_small_workspace(L, entry):
    f = getattr(L, entry)
    args = dict(CALLS[entry], N=100, Cs=65, ldx=65)  # odd rows: copies in the workspace
    rc, n = size(f, args.values())
    assert rc == 0 and n > 0
    small = ctypes.c_size_t(n - 1)
    assert f(*args.values(), at(50), ctypes.byref(small), None) == WORKSPACE
    assert f(*args.values(), at(50) + 16, ctypes.byref(small), None) == UNSUP      # not 256-byte aligned
    assert f(*args.values(), at(50), None, None) == NULL                              # without its size
    big = ctypes.c_size_t(1 << 40)
    out = [k for k in ("y", "dx", "loss") if args.get(k)][0]
    assert f(*dict(args, **{out: at(51)}).values(), at(50), ctypes.byref(big), None) == ALIAS


def test_what_needs_no_workspace(L):
    # one row of aligned arrays: nothing is copied, nothing is split
    args = dict(LINEAR, N=1, Ct=65536, ldy=65536, ldr=65536)
    assert size(L.qcnn_linear_forward, args.values()) == (0, 0)


def test_unread_operands_may_be_null(L):
    args = dict(GRAD, x=None, dw=None, ldx=0)
    assert size(L.qcnn_linear_backward, args.values())[0] == 0
    args = dict(GRAD, w=None, dx=None)
    assert size(L.qcnn_linear_backward, args.values())[0] == 0
    args = dict(GRAD, pre=None, act=0)
    assert size(L.qcnn_linear_backward, args.values())[0] == 0


def test_workspace_of_the_loss_gradient_is_bounded(L):
    # 256 MiB of the logits' gradient, whatever the classes; the rest is small
    for N, Ct in ((4096, 128000), (4096, 1000000), (65536, 128000)):
        args = dict(XGRAD, dtype=BF16, N=N, Cs=1024, ldx=1024, Ct=Ct)
        rc, n = size(L.qcnn_linear_xent_backward, args.values())
        assert rc == 0 and n < (256 << 20) + 4 * N * 1024 + 520 * 4 * 131072 + (1 << 20)


def test_python_refusals():
    x, w, labels = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):  # host tensors
        api.linear_forward(x, w)
    with pytest.raises(ValueError):
        api.gated_forward(x, w)
    with pytest.raises(ValueError):
        api.linear_xent_forward(x, w, labels)
    with pytest.raises(TypeError):
        api.linear_forward(x.double(), w.double())
    with pytest.raises(TypeError):
        api.linear_forward([1.0], w)
    with pytest.raises(ValueError):
        api._act("swish")


def test_sizes_over_many_shapes(L):
    """The host's planning for shapes of every magnitude: an answer, and not
    beyond what copies, 256 MiB of a gradient and split sums come to."""
    import random
    rng = random.Random(5)
    for _ in range(1500):
        entry = rng.choice(list(CALLS))
        dtype, s = rng.choice(((F32, 4), (BF16, 2), (F16, 2)))
        N, Cs, Ct = (int(2 ** rng.uniform(0, b)) for b in (16, 14, 17))
        args = dict(CALLS[entry], dtype=dtype, N=N, Cs=Cs, Ct=Ct)
        for k, cols in (("ldx", Cs), ("ldy", Ct), ("lddy", Ct), ("ldr", Ct)):
            if k in args:
                args[k] = cols + rng.choice((0, 0, 1, 8))
        if any(args.get(k) for k in ("pre", "y", "dx", "dw", "loss")):  # 1 TiB apart: none overlaps
            args = {k: v << 8 if isinstance(v, int) and v >= at(1) else v for k, v in args.items()}
        rc, n = size(getattr(L, entry), args.values())
        assert rc == 0, (entry, args)
        rows = 2 * Ct if "gated" in entry else Ct
        copies = s * ((N + rows) * (Cs + 8) + N * (rows + 8))
        sums = 4 * 513 * rows + 8 * N * (rows // 8 + 64) + 4 * 1024 * 65536 * 2 + 8 * N * (Cs + 8)
        assert n <= copies + sums + (300 << 20), (entry, args, n)
