"""The dense layers (linear, gated, classifying with its loss) on the GPU
against their definitions in float64 on the CPU.

Tolerances, for an output of type T with eps = torch.finfo(T).eps and u =
eps / 2 (half a step, relative):
  * a sum of n products in fp32 is off by at most n 2^-24 A, A the sum of the
    products' magnitudes; in practice roundings do not all have one sign and
    the sums here are folded in blocks: 8 sqrt(n) 2^-24 A is used, and for the
    16-bit types n 2^-24 is below their own rounding;
  * the result is rounded once: u |y|, and the epilogue adds a few fp32
    roundings (16 x 2^-24 of its terms);
  * the backward calls round the products' operand (dz, or the logits'
    gradient) to T once more: u A with A over the rounded operand's products.
"""
import math

import numpy as np
import pytest
import torch

from paper_1512_06473_amd import api

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
E32 = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def half_step(T):
    return torch.finfo(T).eps / 2


def make(seed, T, *shapes, scale=1.0):
    """float64 CPU tensors that T holds exactly."""
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g, dtype=torch.float64) * scale).to(T).double() for s in shapes]


def on(t, T, dev, wider=0):
    """On the GPU in T; wider: as the front columns of rows that much wider,
    with NaN between them."""
    if t is None:
        return None
    if not wider:
        return t.to(T).to(dev)
    big = torch.full((t.shape[0], t.shape[1] + wider), float("nan"), dtype=T, device=dev)
    big[:, :t.shape[1]] = t.to(T).to(dev)
    return big[:, :t.shape[1]]


def value(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope(z, act):
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(value(z, act).sum(), z)[0]


def near(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), "%s: %d of %d over, worst by %g" % (what, int((over > 0).sum()), over.numel(),
                                                                 float(over.max()))


def sum_bound(n, A, T, y, slope_max=1.13):
    """A sum of n products, an activation (of slope at most 1.13) and one rounding."""
    return slope_max * 8 * math.sqrt(n) * E32 * A + half_step(T) * y.abs() + 16 * E32 * (y.abs() + A) + 1e-30 + \
        (2.0 ** -25 if T == torch.float16 else 0)  # fp16's subnormals are 2^-24 apart


SHAPES = [  # N, C_s, C_t
    (1, 1, 1), (1, 64, 128), (1, 4096, 520), (2, 33, 7), (7, 63, 65), (16, 128, 64), (17, 200, 129),
    (128, 64, 128), (129, 136, 257), (300, 1000, 130), (65, 520, 1030), (513, 72, 40),
]


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", SHAPES)
def test_linear_forward(dev, tname, N, Cs, Ct):
    T = TYPES[tname]
    x, w, b, r = make(N + Cs + Ct, T, (N, Cs), (Ct, Cs), (Ct,), (N, Ct))
    z, A = x @ w.t(), x.abs() @ w.abs().t()
    for k, act in enumerate(("none", "relu", "gelu", "gelu_tanh", "silu")):
        bias, res, wider = (b if k % 2 == 0 else None), (r if k in (0, 3) else None), (0, 8, 3, 64, 1)[k]
        zz = z if bias is None else z + bias
        AA = A if bias is None else A + bias.abs()
        y = value(zz, act) if res is None else value(zz, act) + res
        pre = torch.empty(N, Ct, dtype=T, device=dev)
        print("linear_forward", tname, N, Cs, Ct, act, flush=True)
        got = api.linear_forward(on(x, T, dev, wider), on(w, T, dev), on(bias, T, dev), act=act,
                                 residual=on(res, T, dev, wider), pre=pre)
        near(pre, zz, sum_bound(Cs, AA, T, zz), "pre " + act)
        near(got, y, sum_bound(Cs, AA, T, y) + (0 if res is None else 4 * E32 * res.abs()), "y " + act)


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", SHAPES)
def test_linear_backward(dev, tname, N, Cs, Ct):
    T = TYPES[tname]
    u = half_step(T)
    x, w, dy, pre = make(N + Cs + Ct + 1, T, (N, Cs), (Ct, Cs), (N, Ct), (N, Ct))
    for k, act in enumerate(("none", "relu", "gelu", "gelu_tanh", "silu")):
        dz = dy if act == "none" else dy * slope(pre, act)
        wider = (0, 8, 3, 64, 1)[k]
        print("linear_backward", tname, N, Cs, Ct, act, flush=True)
        dx, dw, db = api.linear_backward(on(dy, T, dev, wider), on(x, T, dev, wider), on(w, T, dev), act=act,
                                         pre=None if act == "none" else on(pre, T, dev))
        # dz is rounded to T once (not without an activation); its own fp32 error is a few 2^-24 of dy
        off = (0 if act == "none" else u * dz.abs()) + 16 * E32 * dy.abs() + (2.0 ** -25 if T == torch.float16 else 0)
        near(dx, dz @ w, sum_bound(Ct, dz.abs() @ w.abs(), T, dz @ w) + off @ w.abs(), "dx " + act)
        near(dw, dz.t() @ x, sum_bound(N, dz.t().abs() @ x.abs(), T, dz.t() @ x) + off.t() @ x.abs(), "dw " + act)
        near(db, dz.sum(0), sum_bound(N, dz.abs().sum(0), T, dz.sum(0)) + 16 * E32 * dy.abs().sum(0), "dbias " + act)


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", SHAPES)
def test_gated(dev, tname, N, Cs, Ct):
    T = TYPES[tname]
    uT = half_step(T)
    x, w, b, dy = make(N + Cs + Ct + 2, T, (N, Cs), (2 * Ct, Cs), (2 * Ct,), (N, Ct))
    w = (w / math.sqrt(Cs)).to(T).double()
    z, A = x @ w.t() + b, x.abs() @ w.abs().t() + b.abs()
    for k, act in enumerate(("relu", "gelu", "gelu_tanh", "silu")):
        wider = (0, 8, 3, 1)[k]
        g, u = z[:, :Ct], z[:, Ct:]
        h = value(g, act) * u
        pre = torch.empty(N, 2 * Ct, dtype=T, device=dev)
        print("gated", tname, N, Cs, Ct, act, flush=True)
        xd, wd = on(x, T, dev, wider), on(w, T, dev)
        got = api.gated_forward(xd, wd, on(b, T, dev), act=act, pre=pre)
        near(pre, z, sum_bound(Cs, A, T, z), "pre " + act)
        # each factor's error times the other factor
        eg, eu = 8 * math.sqrt(Cs) * E32 * A[:, :Ct], 8 * math.sqrt(Cs) * E32 * A[:, Ct:]
        near(got, h, sum_bound(1, h.abs(), T, h) + 1.13 * eg * (u.abs() + eu) + eu * value(g, act).abs(), "y " + act)
        p = pre.double().cpu()
        g, u = p[:, :Ct], p[:, Ct:]
        dz = torch.cat([dy * u * slope(g, act), dy * value(g, act)], 1)
        size = torch.cat([dy.abs() * u.abs(), dy.abs() * g.abs()], 1)  # what an fp32 rounding is relative to
        dx, dw, db = api.gated_backward(on(dy, T, dev, wider), xd, wd, pre, act=act)
        off = uT * dz.abs() + 16 * E32 * size + (2.0 ** -25 if T == torch.float16 else 0)
        near(dx, dz @ w, sum_bound(2 * Ct, dz.abs() @ w.abs(), T, dz @ w) + off @ w.abs(), "dx " + act)
        near(dw, dz.t() @ x, sum_bound(N, dz.t().abs() @ x.abs(), T, dz.t() @ x) + off.t() @ x.abs(), "dw " + act)
        near(db, dz.sum(0), sum_bound(N, dz.abs().sum(0), T, dz.sum(0)) + 16 * E32 * size.sum(0), "dbias " + act)


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", SHAPES + [(40, 64, 5000), (700, 96, 2011)])
def test_linear_xent(dev, tname, N, Cs, Ct):
    T = TYPES[tname]
    uT = half_step(T)
    x, w, b = make(N + Cs + Ct + 3, T, (N, Cs), (Ct, Cs), (Ct,))
    w = (2 * w / math.sqrt(Cs)).to(T).double()
    g = torch.Generator().manual_seed(N)
    labels = torch.randint(0, Ct, (N,), generator=g)
    labels[torch.rand(N, generator=g) < 0.2] = -100
    dloss = torch.rand(N, generator=g).float().double() / N
    for bias, wider in ((None, 0), (b, 3)):
        z, A = x @ w.t(), x.abs() @ w.abs().t()
        if bias is not None:
            z, A = z + bias, A + bias.abs()
        lse = torch.logsumexp(z, 1)
        counted = labels >= 0
        at = labels.clamp(min=0)
        loss = torch.where(counted, lse - z.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
        ez = 8 * math.sqrt(Cs) * E32 * A + 4 * E32 * z.abs()  # error of a logit
        e = ez.max(1).values + 32 * E32 * (1 + z.abs().max(1).values)  # exp and log of fp32 arguments
        print("linear_xent", tname, N, Cs, Ct, wider, flush=True)
        xd, wd, ld, bd = on(x, T, dev, wider), on(w, T, dev), labels.to(dev), on(bias, T, dev)
        got, glse = api.linear_xent_forward(xd, wd, ld, bd)
        near(glse, lse, e, "lse")
        near(got, loss, 2 * e + E32 * loss.abs(), "loss")
        assert (got.cpu()[~counted] == 0).all()
        onehot = torch.zeros_like(z).scatter_(1, at[:, None], 1.0)
        weight = torch.where(counted, dloss, torch.zeros_like(dloss))[:, None]
        p = torch.softmax(z, 1)
        d = weight * (p - onehot)
        dx, dw, db = api.linear_xent_backward(dloss.float().to(dev), glse, xd, wd, ld, bd, need_dbias=True)
        # d / max(dloss) is rounded to T (fp16 with a gain of 2^10: its subnormal half step is 2^-35 there)
        off = uT * d.abs() + weight * (p * (2 * e + 32 * E32 * (1 + z.abs().max()))[:, None] + 8 * E32) + \
            (weight > 0) * (2.0 ** -35 * dloss.max() if T == torch.float16 else 0)
        near(dx, d @ w, sum_bound(Ct, d.abs() @ w.abs(), T, d @ w) + off @ w.abs(), "dx")
        near(dw, d.t() @ x, sum_bound(N, d.t().abs() @ x.abs(), T, d.t() @ x) + off.t() @ x.abs(), "dw")
        near(db, d.sum(0), sum_bound(N, d.abs().sum(0), T, d.sum(0)) + off.sum(0), "dbias")
