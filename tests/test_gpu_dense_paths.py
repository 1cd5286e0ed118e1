"""The dense layers' other ways through: sizes that take the large tiles, the
tails of small ones and the split sums; infinities and masks; streams, graphs
and caller-supplied workspaces; rows that stay untouched; and the layers
chained as a feed-forward block and its loss are.

References are float64 (on the GPU, where the sizes are large).  Tolerances as
in test_gpu_dense.py: 8 sqrt(n) 2^-24 of the sum of the products' magnitudes
for an fp32 sum of n products, half a step for a rounding to the type.
"""
import ctypes
import math

import pytest
import torch

from paper_1512_06473_amd import api
from paper_1512_06473_amd._lib import QcnnError, lib

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
    """Within the bound, and infinite exactly where the value rounds to that: a
    type's largest number is (2 - eps) 2^e, and from (2 - eps / 2) 2^e = max +
    half a step on rounding gives infinity (40 x 9000 -> 500 gated in fp16 has
    products of two sums of 9000 terms past 65520)."""
    assert got.shape == want.shape, what
    t = torch.finfo(got.dtype)
    border = t.max * (1 + t.eps / 4)
    assert not torch.isnan(got).any(), what
    over = torch.isinf(got)
    assert (torch.sign(got[over]) == torch.sign(want[over])).all(), what
    assert (want[over].abs() + torch.as_tensor(bound).expand_as(want)[over] >= border).all(), what
    rest = ((got.double() - want).abs() - bound)[~over]
    assert rest.numel() == 0 or float(rest.max()) <= 0, "%s: over by %g" % (what, float(rest.max()))


def product_bound(n, A, y, T):
    return 8 * math.sqrt(n) * E32 * A + torch.finfo(T).eps / 2 * y.abs() + 4 * E32 * y.abs()


# N, C_s, C_t: one round of large tiles; large tiles and a tail along the
# columns; along the rows; small tiles two to a CU; parts of k (few and many)
LARGE = [(4096, 128, 4096), (1999, 136, 17001), (17001, 136, 1999), (2048, 256, 4000), (300, 4096, 200),
         (40, 9000, 1000), (1030, 1000, 1030)]


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", LARGE)
def test_products_of_every_cut(dev, tname, N, Cs, Ct):
    T = TYPES[tname]
    u = torch.finfo(T).eps / 2
    x, w, dy = (normal(dev, T, k, *s) for k, s in ((1, (N, Cs)), (2, (Ct, Cs)), (3, (N, Ct))))
    xd, wd, dyd = x.double(), w.double(), dy.double()
    print("products", tname, N, Cs, Ct, flush=True)
    y = torch.mm(xd, wd.t())
    near(api.linear_forward(x, w), y, product_bound(Cs, torch.mm(xd.abs(), wd.abs().t()), y, T), "y")
    dx, dw, db = api.linear_backward(dy, x, w)
    ref = torch.mm(dyd, wd)
    near(dx, ref, product_bound(Ct, torch.mm(dyd.abs(), wd.abs()), ref, T), "dx")
    ref = torch.mm(dyd.t(), xd)
    near(dw, ref, product_bound(N, torch.mm(dyd.abs().t(), xd.abs()), ref, T), "dw")
    near(db, dyd.sum(0), product_bound(N, dyd.abs().sum(0), dyd.sum(0), T), "dbias")
    half = Ct // 2
    z = y[:, :2 * half]
    A = torch.mm(xd.abs(), wd[:2 * half].abs().t())
    h = api.gated_forward(x, w[:2 * half], act="relu")
    ref = z[:, :half].clamp(min=0) * z[:, half:]
    e = 8 * math.sqrt(Cs) * E32 * A
    near(h, ref, (e[:, :half] * z[:, half:].abs() + e[:, half:] * (z[:, :half].abs() + e[:, :half])) +
         (u + 4 * E32) * ref.abs(), "gated")


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", LARGE[:4] + [(70, 2048, 6000), (3, 64, 40000)])
def test_loss_of_every_cut(dev, tname, N, Cs, Ct):
    T = TYPES[tname]
    x, w, b = normal(dev, T, 1, N, Cs), normal(dev, T, 2, Ct, Cs, scale=2 / math.sqrt(Cs)), normal(dev, T, 3, Ct)
    labels = torch.randint(0, Ct, (N,), generator=torch.Generator().manual_seed(4)).to(dev)
    labels[::7] = -1
    z = torch.mm(x.double(), w.double().t()) + b.double()
    e = (8 * math.sqrt(Cs) * E32 * (torch.mm(x.double().abs(), w.double().abs().t()) + b.double().abs())).max(1).values
    e = e + 32 * E32 * (1 + z.abs().max(1).values)
    lse = torch.logsumexp(z, 1)
    want = torch.where(labels >= 0, lse - z.gather(1, labels.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse))
    print("loss", tname, N, Cs, Ct, flush=True)
    loss, glse = api.linear_xent_forward(x, w, labels, b)
    near(glse, lse, e, "lse")
    near(loss, want, 2 * e + E32 * want.abs(), "loss")


@pytest.mark.parametrize("tname", list(TYPES))
def test_loss_gradient_in_pieces(dev, tname):
    """256 MiB hold 8192 x 16384 (fp32 8192) classes: two pieces and more."""
    T = TYPES[tname]
    N, Cs, Ct = 8192, 64, 20001
    x, w, b = normal(dev, T, 1, N, Cs), normal(dev, T, 2, Ct, Cs, scale=2 / math.sqrt(Cs)), normal(dev, T, 3, Ct)
    labels = torch.randint(0, Ct, (N,), generator=torch.Generator().manual_seed(4)).to(dev)
    labels[5::11] = -100
    weight = torch.where(labels >= 0, 1.0 / N, 0.0)
    loss, lse = api.linear_xent_forward(x, w, labels, b)
    dx, dw, db = api.linear_xent_backward(weight.float(), lse, x, w, labels, b)
    xd, wd = x.double(), w.double()
    z = torch.mm(xd, wd.t()) + b.double()
    d = torch.softmax(z, 1)
    d.scatter_add_(1, labels.clamp(min=0)[:, None], torch.full((N, 1), -1.0, device=dev, dtype=torch.float64))
    d *= weight.double()[:, None]
    # d / weight is rounded to T (fp16: times 2^10, subnormals 2^-24 apart); a logit and lse are off by a few 2^-24
    # of the largest magnitude, exp passes that on
    ez = 64 * E32 * (1 + float(z.abs().max()))
    off = torch.finfo(T).eps / 2 * d.abs() + weight.double()[:, None] * (ez * torch.softmax(z, 1) + 8 * E32 * (d == 0)) + \
        (2.0 ** -35 / N if T == torch.float16 else 0) + E32 / N
    del z
    for got, ref, A, E, n, what in ((dx, torch.mm(d, wd), torch.mm(d.abs(), wd.abs()), torch.mm(off, wd.abs()), Ct, "dx"),
                                    (dw, torch.mm(d.t(), xd), torch.mm(d.abs().t(), xd.abs()),
                                     torch.mm(off.t(), xd.abs()), N, "dw"),
                                    (db, d.sum(0), d.abs().sum(0), off.sum(0), N, "dbias")):
        near(got, ref, product_bound(n, A, ref, T) + E + (2.0 ** -25 if T == torch.float16 else 0), what)


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(dev, act):
    """Directional derivatives of the forward calls in fp32: central
    differences of step h are off by O(h^2) and by the sums' rounding / h."""
    N, Cs, Ct, h = 24, 40, 56, 2.0 ** -6
    x, w, b = normal(dev, torch.float32, 1, N, Cs), normal(dev, torch.float32, 2, 2 * Ct, Cs, scale=0.2), normal(
        dev, torch.float32, 3, 2 * Ct)
    if act == "relu":  # away from the kink: every gate at least 1 from 0
        b[:Ct] = 8.0
    r = normal(dev, torch.float32, 4, N, Ct)
    dirs = [normal(dev, torch.float32, 5 + k, *t.shape) for k, t in enumerate((x, w, b))]

    def gated(s):
        y = api.gated_forward(x + s * dirs[0], w + s * dirs[1], b + s * dirs[2], act=act)
        return float((y.double() * r.double()).sum())

    pre = torch.empty(N, 2 * Ct, device=dev)
    api.gated_forward(x, w, b, act=act, pre=pre)
    grads = api.gated_backward(r, x, w, pre, act=act)
    want = sum(float((g.double() * d.double()).sum()) for g, d in zip(grads, dirs))
    fourth = (8 * (gated(h) - gated(-h)) - (gated(2 * h) - gated(-2 * h))) / (12 * h)
    scale = sum(float((g.double() * d.double()).abs().sum()) for g, d in zip(grads, dirs))
    assert abs(fourth - want) <= 2e-4 * scale, (fourth, want, scale)


@pytest.mark.parametrize("tname", list(TYPES))
def test_rows_of_any_place(dev, tname):
    """Rows that start at odd elements of wider arrays, in and out, with what
    lies between the rows left alone."""
    T = TYPES[tname]
    for N, Cs, Ct in ((5, 40, 24), (70, 130, 66), (300, 64, 128)):
        wide_x, wide_r = normal(dev, T, 1, N, Cs + 5), normal(dev, T, 2, N, Ct + 3)
        flat_w = normal(dev, T, 3, Ct * Cs + 1)
        x, r, w = wide_x[:, 1:1 + Cs], wide_r[:, 3:], flat_w[1:].view(Ct, Cs)
        wide_y = torch.full((N, Ct + 7), 7.0, dtype=T, device=dev)
        y = wide_y[:, 5:5 + Ct]
        api.linear_forward(x, w, residual=r, out=y)
        assert torch.equal(y, api.linear_forward(x.contiguous(), w.clone(), residual=r.contiguous()))
        assert (wide_y[:, :5] == 7).all() and (wide_y[:, 5 + Ct:] == 7).all()
        wide_y[:] = 7
        if Ct % 2 == 0:
            y = wide_y[:, 1:1 + Ct // 2]
            api.gated_forward(x, w, out=y)
            assert torch.equal(y, api.gated_forward(x.contiguous(), w.clone()))
            assert (wide_y[:, :1] == 7).all() and (wide_y[:, 1 + Ct // 2:] == 7).all()
        got = api.linear_backward(r, x, w)
        want = api.linear_backward(r.contiguous(), x.contiguous(), w.clone())
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N", [4, 200])
def test_infinities_and_nan(dev, tname, N):
    """They go where the formula takes them and nowhere else (fp32's products
    of parts would turn an infinity into NaN)."""
    T = TYPES[tname]
    x, w = normal(dev, T, 1, N, 96), normal(dev, T, 2, 150, 96)
    want = torch.mm(x.double(), w.double().t())
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    y = api.linear_forward(x, w)
    keep = [n for n in range(N) if n not in (2, 3)]
    assert torch.isfinite(y[keep]).all()
    assert torch.isnan(y[3]).all()
    assert torch.equal(y[2], torch.copysign(torch.full_like(y[2], float("inf")), w[:, 5]))
    near(y[keep], want[keep], product_bound(96, 96 * 16.0, want[keep], T), "finite rows")
    y = api.linear_forward(x, w, act="relu")
    assert torch.isnan(y[3]).all() and (y[2] == torch.where(w[:, 5] > 0, float("inf"), 0.0)).all()


def test_fp32_keeps_its_range(dev):
    """Sums of numbers near fp32's largest, and of parts of small ones."""
    for scale in (2.0 ** 120, 2.0 ** -60, 2.0 ** -100):
        for N in (8, 100):
            x, w = normal(dev, torch.float32, 1, N, 64), normal(dev, torch.float32, 2, 200, 64)
            x *= scale
            y = api.linear_forward(x, w).double() / scale
            ref = torch.mm(x.double() / scale, w.double().t())
            A = torch.mm(x.double().abs() / scale, w.double().abs().t())
            near(y, ref, 8 * 8 * E32 * A + 4 * E32 * ref.abs(), "scale %g, %d rows" % (scale, N))


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N", [5, 150])
def test_loss_masks_and_labels(dev, tname, N):
    T = TYPES[tname]
    Ct = 300
    x, w, b = normal(dev, T, 1, N, 64), normal(dev, T, 2, Ct, 64, scale=0.2), torch.zeros(Ct, dtype=T, device=dev)
    labels = torch.arange(N, device=dev) % 100
    b[100:] = float("-inf")                       # classes taken out: as if they were not there
    loss, lse = api.linear_xent_forward(x, w, labels, b)
    small, small_lse = api.linear_xent_forward(x, w[:100], labels)
    assert torch.allclose(loss, small, rtol=1e-5, atol=1e-5) and torch.allclose(lse, small_lse, rtol=1e-5, atol=1e-5)
    dloss = torch.full((N,), 1.0 / N, device=dev)
    dx, dw, db = api.linear_xent_backward(dloss, lse, x, w, labels, b)
    assert (dw[100:] == 0).all() and (db[100:] == 0).all() and torch.isfinite(dx).all()
    b[100:] = torch.finfo(T).min                  # the type's lowest value does the same
    low, _ = api.linear_xent_forward(x, w, labels, b)
    assert torch.allclose(low, small, rtol=1e-5, atol=1e-5)
    none = torch.full((N,), -1, device=dev)       # no row counts
    loss, lse = api.linear_xent_forward(x, w, none)
    assert (loss == 0).all() and torch.isfinite(lse).all()
    for g in api.linear_xent_backward(dloss, lse, x, w, none, need_dbias=True):
        assert (g == 0).all()
    over = labels.clone()
    over[1] = Ct                                  # past the classes: NaN, and only there
    loss, lse = api.linear_xent_forward(x, w, over)
    assert torch.isnan(loss[1]) and torch.isfinite(loss[[n for n in range(N) if n != 1]]).all()
    dx, dw, _ = api.linear_xent_backward(dloss, lse, x, w, over)
    assert torch.isnan(dx[1]).all() and torch.isfinite(dx[2:]).all() and torch.isnan(dw).all()


def test_small_loss_weights_in_fp16(dev):
    """1 / N and probabilities of 1e-5 are far below fp16's range together."""
    N, Cs, Ct = 2048, 64, 30000
    x, w = normal(dev, torch.float16, 1, N, Cs), normal(dev, torch.float16, 2, Ct, Cs, scale=0.05)
    labels = torch.randint(0, 100, (N,), generator=torch.Generator().manual_seed(3)).to(dev)
    loss, lse = api.linear_xent_forward(x, w, labels)
    for c in (1.0, 1.0 / N, 2.0 ** -30):
        dx, dw, _ = api.linear_xent_backward(torch.full((N,), c, device=dev), lse, x, w, labels)
        d = torch.softmax(torch.mm(x.double(), w.double().t()), 1)
        d.scatter_add_(1, labels[:, None], torch.full((N, 1), -1.0, device=dev, dtype=torch.float64))
        ref = torch.mm(d.t(), x.double()) * c
        rare = ref[100:]                          # classes that no label names: sums of probabilities alone
        err = float((dw[100:].double() - rare).abs().max())
        # d is rounded to 2^-11 of itself; dw to 2^-11 or fp16's subnormal half step
        assert err <= 2 * 2.0 ** -11 * float((torch.mm(d.abs().t(), x.double().abs())[100:] * c).max()) + 2.0 ** -25, c


def run_all(x, w, wg, wl, dy, labels, dloss):
    pre, pg = torch.empty(x.shape[0], w.shape[0], dtype=x.dtype, device=x.device), torch.empty(
        x.shape[0], wg.shape[0], dtype=x.dtype, device=x.device)
    out = [api.linear_forward(x, w, act="gelu", pre=pre), api.gated_forward(x, wg, pre=pg)]
    out += api.linear_backward(dy, x, w, act="gelu", pre=pre)
    out += api.gated_backward(dy, x, wg, pg)
    loss, lse = api.linear_xent_forward(x, wl, labels)
    return out + [loss, lse] + [g for g in api.linear_xent_backward(dloss, lse, x, wl, labels) if g is not None]


def all_inputs(dev, T, seed, N, Cs, Ct):
    labels = torch.randint(0, 700, (N,), generator=torch.Generator().manual_seed(seed)).to(dev)
    return [normal(dev, T, seed, N, Cs), normal(dev, T, seed + 1, Ct, Cs, scale=0.2),
            normal(dev, T, seed + 2, 2 * Ct, Cs, scale=0.2), normal(dev, T, seed + 3, 700, Cs, scale=0.2),
            normal(dev, T, seed + 4, N, Ct), labels, torch.full((N,), 1.0 / N, device=dev)]


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", [(3, 256, 100), (200, 1000, 130), (129, 65, 77)])
def test_same_results_every_time_and_on_any_stream(dev, tname, N, Cs, Ct):
    ins = all_inputs(dev, TYPES[tname], 1, N, Cs, Ct)
    want = run_all(*ins)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in side:  # two streams at once, a workspace each
        with torch.cuda.stream(s):
            got.append(run_all(*ins))
    torch.cuda.synchronize()
    for g in got + [run_all(*ins)]:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.parametrize("tname", ["fp32", "bf16"])
def test_two_captured_graphs(dev, tname):
    """Graphs captured one after the other, replayed at the same time on two
    streams, on new inputs, with eager work between."""
    T = TYPES[tname]
    shapes = ((200, 1000, 130), (129, 65, 77))  # split sums, copies, sums of columns: every kind of workspace
    sets = [all_inputs(dev, T, 10 * k, *s) for k, s in enumerate(shapes)]
    for ins in sets:
        run_all(*ins)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for ins in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run_all(*ins))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in sets]
    for turn in range(4):
        new = [all_inputs(dev, T, 100 + 10 * turn + k, *s) for k, s in enumerate(shapes)]
        for ins, n in zip(sets, new):
            for a, b in zip(ins, n):
                a.copy_(b)
        want = [run_all(*n) for n in new]
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w)), turn


def test_workspace_of_the_callers_own(dev):
    """The size that the query gives is enough, and nothing behind it is
    touched; the results are those of the library's workspace."""
    x, w = normal(dev, torch.bfloat16, 1, 200, 1001), normal(dev, torch.bfloat16, 2, 130, 1001)
    f, y = lib().qcnn_linear_forward, torch.empty(200, 130, dtype=torch.bfloat16, device=dev)
    args = (1, x.data_ptr(), 1001, 200, 1001, w.data_ptr(), 130, None, 0, None, 0, None, y.data_ptr(), 130)
    stream = torch.cuda.current_stream(dev).cuda_stream
    n = ctypes.c_size_t(0)
    assert f(*args, None, ctypes.byref(n), stream) == 0 and n.value > 0
    room = torch.full((n.value + 4096,), 171, dtype=torch.uint8, device=dev)
    assert f(*args, room.data_ptr(), ctypes.byref(n), stream) == 0
    assert (room[n.value:] == 171).all()
    assert torch.equal(y, api.linear_forward(x, w))


def test_refusals_on_the_gpu(dev):
    x, w = normal(dev, torch.bfloat16, 1, 8, 64), normal(dev, torch.bfloat16, 2, 32, 64)
    labels = torch.zeros(8, dtype=torch.int64, device=dev)
    y = torch.empty(8, 32, dtype=torch.bfloat16, device=dev)
    for call in (lambda: api.linear_forward(x, w.float()), lambda: api.linear_forward(x.double(), w.double()),
                 lambda: api.linear_xent_forward(x, w, labels.int()), lambda: api.linear_xent_forward(x, w, None)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: api.linear_forward(x, w[:, :60]), lambda: api.linear_forward(x.t(), w),
                 lambda: api.linear_forward(x[:1].expand(8, 64), w), lambda: api.linear_forward(x, w, act="swish"),
                 lambda: api.linear_forward(x, w, bias=x[0]), lambda: api.linear_forward(x, w, out=y[:4]),
                 lambda: api.gated_forward(x, w[:31]), lambda: api.linear_forward(x, w.cpu()),
                 lambda: api.linear_backward(y, x, w, need_dx=False, need_dw=False, need_dbias=False),
                 lambda: api.linear_xent_forward(x, w, labels[:4]), lambda: api.linear_forward(x[None], w)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: api.linear_forward(x[:0], w), lambda: api.linear_forward(x, w[:0]),
                 lambda: api.linear_forward(x, w, residual=y, out=y), lambda: api.linear_backward(y, x, w, act="gelu")):
        with pytest.raises(QcnnError):
            call()


def test_feed_forward_block_and_loss(dev):
    """x -> gated layer -> projection with the residual -> loss, forward and
    backward, in bf16 against the same chain in float64 on the same weights;
    every activation is rounded to bf16 between the calls: a few times 2^-8 of
    each gradient's norm."""
    T, N, C, F, V = torch.bfloat16, 333, 512, 1365, 4001
    x, w1, w2, wl = (normal(dev, T, k, *s, scale=c) for k, (s, c) in enumerate(
        [((N, C), 1.0), ((2 * F, C), C ** -0.5), ((C, F), F ** -0.5), ((V, C), 2 * C ** -0.5)]))
    labels = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(9)).to(dev)
    labels[::10] = -100
    weight = torch.where(labels >= 0, 1.0, 0.0) / (labels >= 0).sum()
    pre = torch.empty(N, 2 * F, dtype=T, device=dev)
    h = api.gated_forward(x, w1, pre=pre)
    y = api.linear_forward(h, w2, residual=x)
    loss, lse = api.linear_xent_forward(y, wl, labels)
    dy, dwl, _ = api.linear_xent_backward(weight, lse, y, wl, labels)
    dh, dw2, _ = api.linear_backward(dy, h, w2, need_dbias=False)
    dx, dw1, _ = api.gated_backward(dh, x, w1, pre, need_dbias=False)
    dx = dx + dy  # the residual's gradient
    leaves = [t.double().requires_grad_(True) for t in (x, w1, w2, wl)]
    z = leaves[0] @ leaves[1].t()
    hd = z[:, :F] * torch.sigmoid(z[:, :F]) * z[:, F:]
    logits = (hd @ leaves[2].t() + leaves[0]) @ leaves[3].t()
    lp = torch.log_softmax(logits, 1)
    ref = -(lp.gather(1, labels.clamp(min=0)[:, None])[:, 0] * weight.double()).sum()
    assert abs(float((loss.double() * weight).sum() - ref.detach())) <= 2.0 ** -8 * abs(float(ref.detach()))
    for got, want in zip((dx, dw1, dw2, dwl), torch.autograd.grad(ref, leaves)):
        assert float((got.double() - want).norm()) <= 4 * 2.0 ** -8 * float(want.norm())


def test_responses_of_a_stack_and_its_quantization(dev):
    """The dense layers give quantize_network its targets."""
    from oracle import ec_network
    from paper_1512_06473_amd import quantize_net
    g = torch.Generator().manual_seed(3)
    x = torch.rand(40, 32, generator=g)
    specs = []
    for k, (cs, ct) in enumerate(((32, 24), (24, 16), (16, 10))):
        specs.append({"kind": "fc", "W": torch.randn(ct, cs, generator=g) * 0.3, "relu": k < 2,
                      "bias": torch.randn(ct, generator=g) * 0.1 if k != 1 else None,
                      "D0": torch.randn(cs // 4, 8, 4, generator=g) * 0.3})
    on = [{k: v.to(dev) if isinstance(v, torch.Tensor) else v for k, v in s.items()} for s in specs]
    targets = quantize_net.fc_responses(x.to(dev), on)
    want = ec_network.original_responses(x.numpy(), [{k: v.numpy() if isinstance(v, torch.Tensor) else v
                                                      for k, v in s.items()} for s in specs])
    for t, r in zip(targets, want):
        assert torch.allclose(t.cpu(), torch.from_numpy(r), rtol=1e-5, atol=1e-5)
    got = quantize_net.quantize_network(x.to(dev), on, targets, kmeans_iters=2)
    assert all(float(q["objective"][-1]) <= float(q["objective"][0]) * (1 + 1e-9) for q in got)
    with pytest.raises(ValueError):
        quantize_net.fc_responses(x.to(dev), [{"kind": "pool", "k": 3, "s": 2}])


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", [(40, 2, 6), (40, 66, 30), (300, 1002, 130), (129, 4094, 258), (1030, 1006, 1030),
                                     (4096, 70, 4098)])
def test_rows_that_end_within_16_bytes(dev, tname, N, Cs, Ct):
    """Rows of whole dwords are read in place; what lies behind their ends (NaN
    here, in x, dy and behind the last row) is not."""
    T = TYPES[tname]
    wide_x = torch.full((N, Cs + 2), float("nan"), dtype=T, device=dev)
    wide_dy = torch.full((N, Ct + 2), float("nan"), dtype=T, device=dev)
    flat_w = torch.full((Ct * Cs + 64,), float("nan"), dtype=T, device=dev)
    x, dy, w = wide_x[:, :Cs], wide_dy[:, :Ct], flat_w[:Ct * Cs].view(Ct, Cs)
    x.copy_(normal(dev, T, 1, N, Cs))
    dy.copy_(normal(dev, T, 2, N, Ct))
    w.copy_(normal(dev, T, 3, Ct, Cs))
    xd, wd, dyd = x.double(), w.double(), dy.double()
    print("row ends", tname, N, Cs, Ct, flush=True)
    y = torch.mm(xd, wd.t())
    near(api.linear_forward(x, w), y, product_bound(Cs, torch.mm(xd.abs(), wd.abs().t()), y, T), "y")
    dx, dw, db = api.linear_backward(dy, x, w)
    for got, ref, A, n, what in ((dx, torch.mm(dyd, wd), torch.mm(dyd.abs(), wd.abs()), Ct, "dx"),
                                 (dw, torch.mm(dyd.t(), xd), torch.mm(dyd.abs().t(), xd.abs()), N, "dw"),
                                 (db, dyd.sum(0), dyd.abs().sum(0), N, "dbias")):
        near(got, ref, product_bound(n, A, ref, T), what)
    g = api.gated_forward(x, w, act="relu")
    assert torch.isfinite(g).all()
    labels = torch.arange(N, device=dev) % Ct
    loss, _ = api.linear_xent_forward(x, w, labels)
    assert torch.allclose(loss.double(), torch.logsumexp(y, 1) - y.gather(1, labels[:, None])[:, 0], rtol=1e-4, atol=1e-3)
    # an infinity: fp32's second way, over the same row ends
    x[1, Cs - 1] = float("inf")
    got = api.linear_forward(x, w)
    assert torch.equal(got[1], torch.copysign(torch.full_like(got[1], float("inf")), w[:, Cs - 1]))
    assert torch.isfinite(got[2:]).all()


@pytest.mark.parametrize("tname", ["fp32", "bf16"])
@pytest.mark.parametrize("N", [2500, 8])
def test_rows_past_4_gib(dev, tname, N):
    """Rows 2^20 elements apart, the largest stride: x, dy and y reach behind
    2^32 bytes at 2500 rows (8: the few rows' kernel, the same strides)."""
    T = TYPES[tname]
    Cs, Ct, ld = 72, 40, 1 << 20
    wide = torch.empty(N, ld, dtype=T, device=dev)
    x, dy = wide[:, 1000:1000 + Cs], wide[:, -Ct:]
    x.copy_(normal(dev, T, 1, N, Cs))
    dy.copy_(normal(dev, T, 2, N, Ct))
    w = normal(dev, T, 3, Ct, Cs)
    out = torch.empty(N, ld, dtype=T, device=dev)[:, 17:17 + Ct]
    print("rows past 4 GiB", tname, N, flush=True)
    assert torch.equal(api.linear_forward(x, w, residual=dy, out=out),
                       api.linear_forward(x.contiguous(), w, residual=dy.contiguous()))
    for a, b in zip(api.linear_backward(dy, x, w), api.linear_backward(dy.contiguous(), x.contiguous(), w)):
        assert torch.equal(a, b)
    near(out.contiguous(), torch.mm(x.double(), w.double().t()) + dy.double(),
         product_bound(Cs, torch.mm(x.double().abs(), w.double().abs().t()) + dy.double().abs(), out.double(), T), "y")


@pytest.mark.parametrize("N", [5, 40])
def test_classes_past_4_gib(dev, N):
    """2^20 classes, the most: weights and their gradient reach behind 2^32 bytes."""
    T, Cs, Ct = torch.bfloat16, 2304, 1 << 20
    x, w = normal(dev, T, 1, N, Cs), normal(dev, T, 2, Ct, Cs, scale=1.0 / math.sqrt(Cs))
    labels = torch.randint(Ct - 1000, Ct, (N,), generator=torch.Generator().manual_seed(3)).to(dev)
    xd = x.double()
    z = torch.cat([torch.mm(xd, p.double().t()) for p in w.split(1 << 17)], 1)
    lse = torch.logsumexp(z, 1)
    # a logit is off by 8 sqrt(C_s) 2^-24 of its products' magnitudes, less than sqrt(C_s) standard ones of 1 each
    e = 8 * math.sqrt(Cs) * E32 * math.sqrt(Cs) + 32 * E32 * (1 + float(z.abs().max()))
    print("classes past 4 GiB", N, flush=True)
    loss, glse = api.linear_xent_forward(x, w, labels)
    near(glse, lse, torch.full_like(lse, e), "lse")
    near(loss, lse - z.gather(1, labels[:, None])[:, 0], torch.full_like(lse, 2 * e), "loss")
    dloss = torch.full((N,), 1.0 / N, device=dev)
    dx, dw, _ = api.linear_xent_backward(dloss, glse, x, w, labels)
    last = slice(Ct - 1000, Ct)
    d = torch.softmax(z, 1)
    d.scatter_add_(1, labels[:, None], torch.full((N, 1), -1.0, device=dev, dtype=torch.float64))
    d /= N
    u = 2.0 ** -8  # d and the result are rounded to bf16
    off = u * d.abs() + 2 * e * torch.softmax(z, 1) / N
    for part in (last, slice(0, 1000)):
        dp = d[:, part]
        ref, A = torch.mm(dp.t(), xd), torch.mm(dp.t().abs(), xd.abs())
        near(dw[part], ref, product_bound(N, A, ref, T) + torch.mm(off[:, part].t(), xd.abs()), "dw")
    ref, A, E = (torch.zeros(N, Cs, dtype=torch.float64, device=dev) for _ in range(3))
    for k, p in enumerate(w.split(1 << 17)):
        cols, wd = slice(k << 17, (k + 1) << 17), p.double()
        ref += torch.mm(d[:, cols], wd)
        A += torch.mm(d[:, cols].abs(), wd.abs())
        E += torch.mm(off[:, cols], wd.abs())
    near(dx, ref, product_bound(Ct, A, ref, T) + E, "dx")


@pytest.mark.parametrize("N", [8, 200])
def test_fp32_parts_of_the_smallest_numbers(dev, N):
    """Near 2^-122 the lower parts of a number are subnormal; large weights
    bring the products back to ordinary size.  The parts below 2^-126 are at
    most 2^-126 together, 2^-4 to 2^-24 of the largest, and each of them may be
    dropped by hardware that does not keep subnormals: the sum's bound is then
    C_s 2^-126 |w|."""
    x, w = normal(dev, torch.float32, 1, N, 64), normal(dev, torch.float32, 2, 200, 64)
    x *= 2.0 ** -100
    x[1] *= 2.0 ** -22
    w *= 2.0 ** 90
    y = api.linear_forward(x, w)
    ref = torch.mm(x.double(), w.double().t())
    A = torch.mm(x.double().abs(), w.double().abs().t())
    bound = 8 * 8 * E32 * A + 4 * E32 * ref.abs()
    bound[1] += 2.0 ** -126 * w.double().abs().sum(1)
    near(y, ref, bound, "small numbers")


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N,Cs,Ct", [(8, 72, 40), (300, 200, 130), (1030, 1000, 1030)])
def test_what_lies_between_rows_decides_nothing(dev, tname, N, Cs, Ct):
    """Bit for bit the same results with NaN, infinities or zeros there."""
    T = TYPES[tname]
    w, results = normal(dev, T, 3, Ct, Cs), []
    for fill in (0.0, float("nan"), float("inf")):
        wide_x = torch.full((N, Cs + 64), fill, dtype=T, device=dev)
        wide_dy = torch.full((N, Ct + 64), fill, dtype=T, device=dev)
        x, dy = wide_x[:, 8:8 + Cs], wide_dy[:, 16:16 + Ct]
        x.copy_(normal(dev, T, 1, N, Cs))
        dy.copy_(normal(dev, T, 2, N, Ct))
        results.append([api.linear_forward(x, w, residual=dy), api.gated_forward(x, w), *api.linear_backward(dy, x, w)])
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N", [1, 15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("Cs,Ct", [(1, 1), (127, 31), (129, 4100), (1025, 333), (5000, 20)])
def test_weight_gradients_of_few_rows(dev, tname, N, Cs, Ct):
    """Both sides of the switch between the kernels, odd sizes, rows of x and dy
    at odd places; and the guard behind dw stays as it was."""
    T = TYPES[tname]
    wide_x = torch.full((N, Cs + 3), float("nan"), dtype=T, device=dev)
    wide_dy = torch.full((N, Ct + 5), float("nan"), dtype=T, device=dev)
    x, dy = wide_x[:, 1:1 + Cs], wide_dy[:, 3:3 + Ct]
    x.copy_(normal(dev, T, 1, N, Cs))
    dy.copy_(normal(dev, T, 2, N, Ct))
    print("few rows", tname, N, Cs, Ct, flush=True)
    flat = torch.full((Ct * Cs + 64,), 7.0, dtype=T, device=dev)
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[T]
    rc = lib().qcnn_linear_backward(code, dy.data_ptr(), Ct + 5, x.data_ptr(), Cs + 3, N, Cs, None, Ct, None, 0, None,
                                    flat.data_ptr(), None, None, None, torch.cuda.current_stream(dev).cuda_stream)
    assert rc == 0
    ref, A = torch.mm(dy.double().t(), x.double()), torch.mm(dy.double().abs().t(), x.double().abs())
    # below 2^-14 fp16's numbers are 2^-24 apart: half a step is 2^-25, not 2^-11 of the value
    bound = product_bound(N, A, ref, T) + (2.0 ** -25 if T == torch.float16 else 0)
    near(flat[:Ct * Cs].view(Ct, Cs), ref, bound, "dw")
    assert (flat[Ct * Cs:] == 7).all()


@pytest.mark.parametrize("tname", list(TYPES))
@pytest.mark.parametrize("N", [1, 16, 17, 32, 33])
@pytest.mark.parametrize("Cs,Ct", [(1, 1), (31, 127), (63, 4099), (333, 1025), (4100, 129), (70, 20000)])
def test_input_gradients_of_few_rows(dev, tname, N, Cs, Ct):
    """The same for dx, with NaN behind the last weight and the last dy."""
    T = TYPES[tname]
    wide_dy = torch.full((N, Ct + 5), float("nan"), dtype=T, device=dev)
    flat_w = torch.full((Ct * Cs + 64,), float("nan"), dtype=T, device=dev)
    dy, w = wide_dy[:, 3:3 + Ct], flat_w[:Ct * Cs].view(Ct, Cs)
    dy.copy_(normal(dev, T, 1, N, Ct))
    w.copy_(normal(dev, T, 2, Ct, Cs))
    print("few rows dx", tname, N, Cs, Ct, flush=True)
    flat = torch.full((N * Cs + 64,), 7.0, dtype=T, device=dev)
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[T]
    rc = lib().qcnn_linear_backward(code, dy.data_ptr(), Ct + 5, None, 0, N, Cs, w.data_ptr(), Ct, None, 0,
                                    flat.data_ptr(), None, None, None, None, torch.cuda.current_stream(dev).cuda_stream)
    assert rc == 0
    ref, A = torch.mm(dy.double(), w.double()), torch.mm(dy.double().abs(), w.double().abs())
    # below 2^-14 fp16's numbers are 2^-24 apart: half a step is 2^-25, not 2^-11 of the value
    bound = product_bound(Ct, A, ref, T) + (2.0 ** -25 if T == torch.float16 else 0)
    near(flat[:N * Cs].view(N, Cs), ref, bound, "dx")
    assert (flat[N * Cs:] == 7).all()
