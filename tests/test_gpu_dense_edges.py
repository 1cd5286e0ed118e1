"""The dense layers where numbers run out: NaN among a row's logits, loss
weights and activations at the ends of their range, fp32's accuracy in one
sign, gradients of a size that a 16-bit type still holds, and the largest
sizes.

References are float64; tolerances count half steps of 2^-24 (fp32) or of the
type, as in test_gpu_dense.py, and are derived at each test.
"""
import math

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


def normal(dev, T, seed, *shape, scale=1.0):
    g = torch.Generator(device=dev).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=dev) * scale).to(T)


def near(got, want, bound, what):
    assert got.shape == want.shape, what
    assert torch.isfinite(got).all(), what
    over = float(((got.double() - want).abs() - bound).max())
    assert over <= 0, "%s: over by %g" % (what, over)


# N, C_s, C_t: few rows by 16 and by 32 columns a wave (fp32: 20 rows too);
# small tiles; large ones and a tail; parts of k whose sums one workgroup a row
# finishes, and several
LOSSES = [(4, 64, 301), (13, 64, 16401), (20, 64, 301), (300, 64, 257), (1999, 136, 17001), (40, 4096, 257),
          (70, 2048, 6001)]


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", LOSSES)
def test_nan_logits_reach_the_loss(dev, tname, N, Cs, Ct):
    """Whichever class has them, and whatever its neighbours are: all of a
    lane's, a quad's or a tile's classes NaN or masked, and others finite."""
    T = TYPES[tname]
    x, w = normal(dev, T, 1, N, Cs), normal(dev, T, 2, Ct, Cs, scale=1 / math.sqrt(Cs))
    labels = torch.arange(N, device=dev) % 7 + 8  # no label is a class that is NaN or masked below
    labels[1] = -1
    counted = labels >= 0
    nan, gone = float("nan"), float("-inf")
    places = [0, 1, 2, 3, 4, 16, 17, 19, 64, 255, 256, Ct - 2, Ct - 1]
    for c in places:
        for masked in ((), (slice(max(0, c - c % 4), c), slice(c + 1, c + 4)), (slice(20, None),), (slice(1, 8),)):
            bias = torch.zeros(Ct, dtype=T, device=dev)
            for m in masked:
                bias[m] = gone
            bias[c] = nan
            print("nan", tname, N, Cs, Ct, c, masked, flush=True)
            loss, lse = api.linear_xent_forward(x, w, labels, bias)
            assert torch.isnan(lse).all() and torch.isnan(loss[counted]).all() and loss[1] == 0, (c, masked)
    for rows in (slice(0, 1), slice(3, 4), slice(Ct - 1, Ct), slice(16, min(Ct, 16 + 512)), slice(Ct - 200, Ct)):
        bad = w.clone()
        bad[rows] = nan
        loss, lse = api.linear_xent_forward(x, bad, labels)
        assert torch.isnan(lse).all() and torch.isnan(loss[counted]).all() and loss[1] == 0, rows
    dx, dw, db = api.linear_xent_backward(torch.full((N,), 1.0 / N, device=dev), lse, x, w, labels, need_dbias=True)
    assert torch.isnan(dx[counted]).all() and (dx[1] == 0).all() and torch.isnan(dw).all() and torch.isnan(db).all()
    bias = torch.zeros(Ct, dtype=T, device=dev)
    bias[Ct - 1] = float("inf")  # inf - inf
    loss, lse = api.linear_xent_forward(x, w, labels, bias)
    assert torch.isnan(lse).all() and torch.isnan(loss[counted]).all() and loss[1] == 0
    # a row of x: that row alone
    x[2, 3] = nan
    loss, lse = api.linear_xent_forward(x, w, labels)
    keep = torch.arange(N, device=dev) != 2
    assert torch.isnan(lse[2]) and torch.isnan(loss[2])
    assert torch.isfinite(lse[keep]).all() and torch.isfinite(loss[keep]).all()


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", LOSSES)
def test_classes_masked_all_but_one(dev, tname, N, Cs, Ct):
    """The joins of empty sets with the one that is left: its logit is lse."""
    T = TYPES[tname]
    x, w = normal(dev, T, 1, N, Cs), normal(dev, T, 2, Ct, Cs, scale=1 / math.sqrt(Cs))
    for c in (0, 3, 130, Ct - 1):
        bias = torch.full((Ct,), float("-inf"), dtype=T, device=dev)
        bias[c] = 0
        loss, lse = api.linear_xent_forward(x, w, torch.full((N,), c, device=dev), bias)
        z = torch.mm(x.double(), w[c:c + 1].double().t())[:, 0]
        # a sum of C_s products, then log(1) = 0 is added
        A = torch.mm(x.double().abs(), w[c:c + 1].double().abs().t())[:, 0]
        near(lse, z, 8 * math.sqrt(Cs) * E32 * A + 2 * E32 * z.abs(), "lse")
        assert (loss == 0).all()


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N", [4, 200])
def test_nan_and_infinities_in_the_gated_layer(dev, tname, N):
    """They go where the formula takes them and nowhere else."""
    T = TYPES[tname]
    x, w = normal(dev, T, 1, N, 96), normal(dev, T, 2, 2 * 75, 96, scale=0.1)
    z, A = torch.mm(x.double(), w.double().t()), torch.mm(x.double().abs(), w.double().abs().t())
    gate, up = z[:, :75] * torch.sigmoid(z[:, :75]), z[:, 75:]
    want, e = gate * up, 8 * math.sqrt(96) * E32 * A
    # each factor's error times the other factor, silu's slope at most 1.1; one rounding (fp16: or half of 2^-24)
    bound = 1.1 * e[:, :75] * (up.abs() + e[:, 75:]) + e[:, 75:] * gate.abs() + 16 * E32 * z[:, :75].abs() * up.abs() + \
        torch.finfo(T).eps / 2 * want.abs() + (2.0 ** -25 if T == torch.float16 else 0)
    x[2, 5] = float("nan")
    x[3, 7] = float("inf")
    w2 = w.clone()
    w2[10, 1], w2[75 + 20, 2] = float("nan"), float("inf")
    keep = [n for n in range(N) if n not in (2, 3)]
    y = api.gated_forward(x, w)
    assert torch.isnan(y[2]).all() and not torch.isfinite(y[3]).any()
    near(y[keep], want[keep], bound[keep], "rows")
    y = api.gated_forward(x, w2)
    assert torch.isnan(y[:, 10]).all() and not torch.isfinite(y[:, 20]).any()
    cols = [c for c in range(75) if c not in (10, 20)]
    near(y[keep][:, cols], want[keep][:, cols], bound[keep][:, cols], "columns")


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N", [6, 150])
@pytest.mark.parametrize("c", [2.0 ** -100, 2.0 ** -119, 2.0 ** -127, 2.0 ** -140])
def test_smallest_loss_weights(dev, tname, N, c):
    """Weights whose reciprocal no float holds, beside rows of weight 0 and
    rows left out.  Large x (small w: logits of ordinary size) bring dw back
    into fp32's and bf16's normal range; all of fp16's gradients round to 0."""
    T = TYPES[tname]
    up = 1.0 if T == torch.float16 else 2.0 ** 60
    Cs, Ct = 64, 90
    x, w = normal(dev, T, 1, N, Cs, scale=up), normal(dev, T, 2, Ct, Cs, scale=1 / (8 * up))
    labels = torch.arange(N, device=dev) % Ct
    labels[4] = -1
    weight = torch.full((N,), c, device=dev)
    weight[1::2] = 0.0
    _, lse = api.linear_xent_forward(x, w, labels)
    dx, dw, db = api.linear_xent_backward(weight, lse, x, w, labels, need_dbias=True)
    for g in (dx, dw, db):
        assert torch.isfinite(g).all()
    if T == torch.float16:
        assert (dx == 0).all() and (dw == 0).all() and (db == 0).all()
        return
    z = torch.mm(x.double(), w.double().t())
    p = torch.softmax(z, 1)
    d = p.clone()
    d[torch.arange(N, device=dev), labels.clamp(min=0)] -= 1.0
    on = torch.where(labels >= 0, weight.double(), torch.zeros(N, dtype=torch.float64, device=dev))[:, None]
    d = d * on
    # a logit is off by its sum's rounding, lse too, and exp passes that on; d is rounded to T once
    ez = 8 * math.sqrt(Cs) * E32 * torch.mm(x.double().abs(), w.double().abs().t()).max(1).values[:, None] + 64 * E32
    off = torch.finfo(T).eps / 2 * d.abs() + on * (2 * ez * p + 8 * E32)
    ref, A = torch.mm(d.t(), x.double()), torch.mm(d.t().abs(), x.double().abs())
    near(dw, ref, (8 * math.sqrt(N) + 4) * E32 * A + torch.finfo(T).eps / 2 * ref.abs() + torch.mm(off.t(), x.double().abs()),
         "dw")
    # what is left of dbias and dx is subnormal or 0: within one smallest normal number
    near(db, d.sum(0), off.sum(0) + 2 * torch.finfo(T).eps * d.abs().sum(0) + 2.0 ** -126, "dbias")
    near(dx, torch.mm(d, w.double()), torch.full((N, Cs), 2.0 ** -126, dtype=torch.float64, device=dev), "dx")


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Ct", [(1, 1), (11, 77), (32, 1000), (33, 513), (700, 130)])
def test_bias_gradients_alone(dev, tname, N, Ct):
    """The same bits as beside the products."""
    T = TYPES[tname]
    x, w, dy, pre = (normal(dev, T, k, *s) for k, s in enumerate([(N, 65), (2 * Ct, 65), (N, Ct), (N, 2 * Ct)]))
    for act in ("none", "relu", "gelu", "gelu_tanh", "silu"):
        alone = api.gated_backward(dy, x, w, pre, act=act, need_dx=False, need_dw=False)
        assert alone[0] is None and alone[1] is None
        assert torch.equal(alone[2], api.gated_backward(dy, x, w, pre, act=act)[2])
        half = pre[:, :Ct].contiguous()
        alone = api.linear_backward(dy, x, w[:Ct], act=act, pre=half, need_dx=False, need_dw=False)
        assert torch.equal(alone[2], api.linear_backward(dy, x, w[:Ct], act=act, pre=half)[2])


@pytest.mark.parametrize("n", [1, 2, 4])
def test_fp32_products_of_one_sign(dev, n):
    """Numbers just below 1 + 2^-7: were their upper 8 bits cut off, 16 bits of
    each would be left, and the smallest products of the parts, which are left
    out, would come to 8 x 2^-24 of a product, always of one sign.  Rounded to
    the nearest 8 bits they are 1 + 2^-7 less 2^-23, with nothing left out.  Of
    n = 1, 2 or 4 equal products every partial sum up to the last addition is
    exact or below 2^-21 of the whole: off by half a step at the end, 2^-24, or
    a whole one if the matrix cores cut off, and 2^-44: within 3 x 2^-24."""
    v = 1 + 2.0 ** -7 - 2.0 ** -23
    N, C = 70, 130
    for sign in (1.0, -1.0):
        x, w = torch.zeros(N, C, device=dev), torch.zeros(150, C, device=dev)
        x[:, :n], w[:, :n] = v, sign * v
        want = torch.full((N, 150), n * sign * v * v, dtype=torch.float64, device=dev)
        near(api.linear_forward(x, w), want, 3 * E32 * want.abs(), "y")
        dy, w = torch.zeros(N, 150, device=dev), torch.full((150, C), v, device=dev)
        dy[:, 100:100 + n] = sign * v
        dx, _, _ = api.linear_backward(dy, x, w, need_dw=False)
        want = torch.full((N, C), n * sign * v * v, dtype=torch.float64, device=dev)
        near(dx, want, 3 * E32 * want.abs(), "dx")
        dy, x = torch.zeros(N, 150, device=dev), torch.full((N, C), v, device=dev)
        dy[60:60 + n] = sign * v
        _, dw, _ = api.linear_backward(dy, x, w, need_dx=False)
        want = torch.full((150, C), n * sign * v * v, dtype=torch.float64, device=dev)
        near(dw, want, 3 * E32 * want.abs(), "dw")


def test_fp32_largest_numbers(dev):
    """Up to the largest there is, whose upper bits round to an infinity: as
    exact as any other, in ordinary sums."""
    top = torch.finfo(torch.float32).max
    for N in (8, 70):
        x, w = normal(dev, torch.float32, 1, N, 40), normal(dev, torch.float32, 2, 150, 40, scale=2.0 ** -6)
        x[1, 3], x[2, 4] = top, -top
        w[:, 3:5] *= 2.0 ** -4
        y, ref = api.linear_forward(x, w), torch.mm(x.double(), w.double().t())
        A = torch.mm(x.double().abs(), w.double().abs().t())
        near(y, ref, 8 * math.sqrt(40) * E32 * A + E32 * ref.abs(), "%d rows" % N)


@pytest.mark.parametrize("N", [8, 40])
def test_gelu_of_negative_numbers_in_fp32(dev, N):
    """Phi(z) far down its tail, to a few steps of itself (1 + erf would leave
    nothing below -5.5).  z / sqrt(2) is off by 1.5 half steps, and the tail
    passes on 1 + z^2 times that; the function itself is good to 16 steps."""
    z = torch.linspace(-12.0, 6.0, 3001, device=dev)
    zd = z.double()
    phi = 0.5 * torch.special.erfc(-zd / math.sqrt(2.0))
    steps = 1.5 * zd * zd + 48
    y = api.linear_forward(torch.ones(N, 1, device=dev), z[:, None].contiguous(), act="gelu")
    near(y, (zd * phi).expand(N, -1), (steps * E32 * (zd * phi).abs()).expand(N, -1), "gelu")
    dx, _, _ = api.linear_backward(torch.ones(3001, 1, device=dev), z[:, None], torch.ones(1, 1, device=dev), act="gelu",
                                   pre=z[:, None].contiguous(), need_dw=False, need_dbias=False)
    density = torch.exp(-0.5 * zd * zd) / math.sqrt(2.0 * math.pi)
    near(dx[:, 0], phi + zd * density, steps * E32 * (phi + (zd * density).abs()), "slope")


@pytest.mark.parametrize("tname", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_of_the_largest_numbers(dev, tname, act):
    """From where z^2 overflows up to the largest number: z and 0, slopes 1 and 0."""
    T = TYPES[tname]
    z = torch.tensor([1e13, 1e18, 3e19, 1e20, 1e30, float(torch.finfo(T).max)], dtype=torch.float64).to(T).to(dev)
    z = torch.cat([z, -z])[:, None].contiguous()
    one, up = torch.ones(1, 1, dtype=T, device=dev), (z > 0).double()
    for N in (12, 60):  # few rows, and tiles
        zz = z.repeat(N // 12, 1)
        y = api.linear_forward(zz, one, act=act)
        assert torch.equal(y.double(), zz.double() * up.repeat(N // 12, 1)), act
        dx, _, db = api.linear_backward(torch.ones_like(zz), zz, one, act=act, pre=zz, need_dw=False)
        assert torch.equal(dx.double(), up.repeat(N // 12, 1)) and float(db) == N / 2, act
        g = torch.cat([zz, torch.ones_like(zz)], 1)
        w2 = torch.ones(2, 1, dtype=T, device=dev)
        dx, _, db = api.gated_backward(torch.full_like(zz, 2.0 ** -64), zz, w2, g, act=act, need_dw=False)
        assert torch.isfinite(dx).all() and float(db[0]) == N / 2 * 2.0 ** -64, act


def test_small_loss_weights_in_fp16_by_value(dev):
    """A weight of 2^-30 in fp16, with x or w so large that the gradients are
    numbers that fp16 holds: all zeros would not do."""
    T, c, N, Cs, Ct = torch.float16, 2.0 ** -30, 4096, 64, 40
    for big_x in (True, False):
        up = 2.0 ** 13
        x = normal(dev, T, 1, N, Cs, scale=up if big_x else 1 / up)
        w = normal(dev, T, 2, Ct, Cs, scale=(1 / up if big_x else up) / 8)
        labels = torch.randint(0, Ct, (N,), generator=torch.Generator().manual_seed(3)).to(dev)
        _, lse = api.linear_xent_forward(x, w, labels)
        dx, dw, _ = api.linear_xent_backward(torch.full((N,), c, device=dev), lse, x, w, labels)
        xd, wd = x.double(), w.double()
        z = torch.mm(xd, wd.t())
        p = torch.softmax(z, 1)
        d = p.clone()
        d[torch.arange(N, device=dev), labels] -= 1.0
        d *= c
        ez = 8 * math.sqrt(Cs) * E32 * torch.mm(xd.abs(), wd.abs().t()).max(1).values[:, None] + \
            64 * E32 * (1 + z.abs().max())
        # d / c is rounded to fp16 (times 2^10: subnormal half steps of 2^-35), the result too (2^-25)
        off = 2.0 ** -11 * d.abs() + c * (2 * ez * p + 8 * E32 + 2.0 ** -35)
        for got, ref, A, E, n, used in ((dw, torch.mm(d.t(), xd), torch.mm(d.abs().t(), xd.abs()),
                                         torch.mm(off.t(), xd.abs()), N, big_x),
                                        (dx, torch.mm(d, wd), torch.mm(d.abs(), wd.abs()), torch.mm(off, wd.abs()), Ct,
                                         not big_x)):
            if used:
                bound = 8 * math.sqrt(n) * E32 * A + 2.0 ** -11 * ref.abs() + E + 2.0 ** -25
                assert float((ref.abs() - bound).max()) > 0  # zeros would fail
                near(got, ref, bound, "dw" if big_x else "dx")


# One round of large tiles; parts of k; odd widths, so that dz's two halves
# end within 16 bytes
GATED = [(4096, 136, 2048), (2048, 256, 2000), (1030, 1000, 1031), (300, 2000, 77), (513, 520, 4003)]


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("N,Cs,Ct", GATED)
def test_gated_gradients_of_every_cut(dev, tname, act, N, Cs, Ct):
    T = TYPES[tname]
    u = torch.finfo(T).eps / 2
    x, w = normal(dev, T, 1, N, Cs), normal(dev, T, 2, 2 * Ct, Cs, scale=1 / math.sqrt(Cs))
    dy, pre = normal(dev, T, 3, N, Ct), normal(dev, T, 4, N, 2 * Ct)
    g, up, d = pre[:, :Ct].double(), pre[:, Ct:].double(), dy.double()
    phi = 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) if act == "gelu" else torch.sigmoid(g)
    value = g * phi
    slope = phi + g * (torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi) if act == "gelu" else phi * (1 - phi))
    dz = torch.cat([d * up * slope, d * value], 1)
    size = torch.cat([d.abs() * up.abs(), d.abs() * g.abs()], 1)  # what an fp32 rounding is relative to
    off = u * dz.abs() + 16 * E32 * size + (2.0 ** -25 if T == torch.float16 else 0)
    print("gated gradients", tname, act, N, Cs, Ct, flush=True)
    dx, dw, db = api.gated_backward(dy, x, w, pre, act=act)
    xd, wd = x.double(), w.double()
    tiny = 2.0 ** -25 if T == torch.float16 else 0

    def bound(n, A, ref):
        return 8 * math.sqrt(n) * E32 * A + u * ref.abs() + 16 * E32 * ref.abs() + tiny

    ref = torch.mm(dz, wd)
    near(dx, ref, bound(2 * Ct, torch.mm(dz.abs(), wd.abs()), ref) + torch.mm(off, wd.abs()), "dx")
    ref = torch.mm(dz.t(), xd)
    near(dw, ref, bound(N, torch.mm(dz.abs().t(), xd.abs()), ref) + torch.mm(off.t(), xd.abs()), "dw")
    near(db, dz.sum(0), bound(N, dz.abs().sum(0), dz.sum(0)) + 16 * E32 * size.sum(0), "dbias")


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", [(1 << 21, 8, 18), (1 << 21, 7, 5), (4, 1 << 20, 6), (40, 1 << 20, 6),
                                     (4, 6, 1 << 20), (40, 6, 1 << 20)])
def test_the_largest_sizes(dev, tname, N, Cs, Ct):
    """2^21 rows, 2^20 columns: every call at the limits that the header names."""
    T = TYPES[tname]
    u = torch.finfo(T).eps / 2
    tiny = 2.0 ** -25 if T == torch.float16 else 0  # half of fp16's smallest number
    big = max(N, Cs, Ct) ** -0.25                   # keeps fp16's sums of 2^21 terms in range
    x, w, dy = (normal(dev, T, k, *s, scale=big) for k, s in enumerate([(N, Cs), (Ct, Cs), (N, Ct)]))
    xd, wd, dyd = x.double(), w.double(), dy.double()
    print("largest", tname, N, Cs, Ct, flush=True)

    def bound(n, a, b, ref):
        return 8 * math.sqrt(n) * E32 * torch.mm(a.abs(), b.abs()) + (u + 4 * E32) * ref.abs() + tiny

    ref = torch.mm(xd, wd.t())
    near(api.linear_forward(x, w), ref, bound(Cs, xd, wd.t(), ref), "y")
    half = Ct // 2
    if half * 2 == Ct:
        e = bound(Cs, xd, wd.t(), ref) - (u + 4 * E32) * ref.abs() - tiny
        g, up = ref[:, :half], ref[:, half:]
        want = g.clamp(min=0) * up
        near(api.gated_forward(x, w, act="relu"), want,
             e[:, :half] * (up.abs() + e[:, half:]) + e[:, half:] * g.abs() + (u + 8 * E32) * want.abs() + tiny, "gated")
    dx, dw, db = api.linear_backward(dy, x, w)
    ref = torch.mm(dyd, wd)
    near(dx, ref, bound(Ct, dyd, wd, ref), "dx")
    ref = torch.mm(dyd.t(), xd)
    near(dw, ref, bound(N, dyd.t(), xd, ref), "dw")
    ref = dyd.sum(0)
    near(db, ref, 8 * math.sqrt(N) * E32 * dyd.abs().sum(0) + (u + 4 * E32) * ref.abs() + tiny, "dbias")
    del ref
    labels = torch.arange(N, device=dev) % Ct
    z = torch.mm(xd, wd.t())
    lse = torch.logsumexp(z, 1)
    loss, glse = api.linear_xent_forward(x, w, labels)
    ez = 8 * math.sqrt(Cs) * E32 * torch.mm(xd.abs(), wd.abs().t()).max(1).values + 32 * E32 * (1 + z.abs().max() + lse.abs())
    near(glse, lse, ez, "lse")
    near(loss, lse - z.gather(1, labels[:, None])[:, 0], 2 * ez + E32 * lse.abs(), "loss")
    gx, gw, gb = api.linear_xent_backward(torch.full((N,), 1.0, device=dev), glse, x, w, labels, need_dbias=True)
    p = torch.softmax(z, 1)
    d = p.clone()
    d.scatter_add_(1, labels[:, None], torch.full((N, 1), -1.0, device=dev, dtype=torch.float64))
    # d is rounded to T (fp16: times 2^10, subnormal half steps 2^-35); logits and lse are off by ez each
    off = u * d.abs() + p * (2 * ez)[:, None] + 8 * E32 * d.abs() + (2.0 ** -35 if T == torch.float16 else 0)
    ref = torch.mm(d, wd)
    near(gx, ref, bound(Ct, d, wd, ref) + torch.mm(off, wd.abs()), "loss dx")
    ref = torch.mm(d.t(), xd)
    near(gw, ref, bound(N, d.t(), xd, ref) + torch.mm(off.t(), xd.abs()), "loss dw")
    ref = d.sum(0)
    near(gb, ref, 8 * math.sqrt(N) * E32 * d.abs().sum(0) + (u + 4 * E32) * ref.abs() + off.sum(0) + tiny, "loss dbias")


def test_two_threads_on_one_stream(dev):
    """Calls that share the stream's workspace (copies, split sums, sums of
    columns), enqueued by two threads at once: each as if it were alone."""
    import threading
    jobs = []
    for k, (N, Cs, Ct) in enumerate([(200, 1001, 130), (129, 65, 77)]):
        x, w, dy = (normal(dev, torch.bfloat16, 3 * k + i, *s) for i, s in enumerate([(N, Cs), (Ct, Cs), (N, Ct)]))
        jobs.append((x, w, dy, [api.linear_forward(x, w), *api.linear_backward(dy, x, w)]))
    torch.cuda.synchronize()
    wrong = []

    def work(x, w, dy, want):
        for _ in range(40):
            got = [api.linear_forward(x, w), *api.linear_backward(dy, x, w)]
            torch.cuda.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)):
                wrong.append(tuple(x.shape))

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
