"""Performance cases of the dense fully-connected operators: the linear layer,
the gated feed-forward layer and the classifying layer with its softmax cross
entropy, forward and backward.

A case is a dict of plain values.  ``listed()`` gives the fixed ones and
``draw(rng)`` one more of the same ranges; ``prepare(case, seed)`` makes what a
program holds before the call, ``run(state)`` is one pass, ``work(case)`` the
bytes and operations that the pass cannot do without, and ``exact(case, seed)``
the result in float64.  ``run`` computes the plain form of each operator in
elementary torch operations, or, with ``own`` set, through this package.

Sizes: N rows (tokens, images), C_s input channels, C_t output channels (the
gated layer has 2 C_t weight rows, gate first; the loss has C_t classes).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def case(name, op, type_, N, Cs, Ct, act="none", bias=False, residual=False, strided=False):
    """op: linear, linear_grad, gated, gated_grad, loss, loss_grad; strided:
    the rows of x are the front part of wider rows."""
    return {**({"name": name} if name else {}), "op": op, "type": type_, "N": N, "Cs": Cs, "Ct": Ct, "act": act,
            "bias": bias, "residual": residual, "strided": strided}


def listed():
    return [
        # One new token through an output projection that adds to the residual stream.
        case("linear_1_token", "linear", "bf16", 1, 4096, 4096, bias=True, residual=True),
        # The fc6 layer of the AlexNet-shaped network before it is quantized, a batch.
        case("linear_fc6_n128_fp32", "linear", "fp32", 128, 9216, 4096, act="relu", bias=True),
        # A long prompt through the first product of a feed-forward block.
        case("linear_prompt_8192", "linear", "bf16", 8192, 4096, 16384, act="gelu_tanh", bias=True),
        # Training a square projection on a batch of tokens.
        case("linear_grad_4096_fp16", "linear_grad", "fp16", 4096, 4096, 4096, act="gelu", bias=True),
        # Training a small layer of odd sizes in full precision.
        case("linear_grad_odd_fp32", "linear_grad", "fp32", 1001, 1537, 2049, act="silu", bias=True),
        # A few sequences decoded together, a token each.
        case("gated_8_tokens", "gated", "bf16", 8, 4096, 11008, act="silu"),
        # A short prompt through a small layer of odd sizes, rows cut out of wider ones.
        case("gated_odd_fp16", "gated", "fp16", 333, 1000, 2731, act="gelu", bias=True, strided=True),
        # A long prompt through a gated feed-forward block.
        case("gated_prompt_8192", "gated", "bf16", 8192, 4096, 11008, act="silu"),
        # Training that block on a batch of tokens.
        case("gated_grad_4096", "gated_grad", "bf16", 4096, 4096, 11008, act="silu"),
        # The loss of the AlexNet-shaped network's last layer on a batch.
        case("loss_fc8_n64_fp32", "loss", "fp32", 64, 4096, 1000, bias=True),
        # Scoring a text with a vocabulary of odd size.
        case("loss_1999_odd", "loss", "bf16", 1999, 2048, 50001),
        # Training the last layer of a language model with a large vocabulary.
        case("loss_grad_4096", "loss_grad", "bf16", 4096, 4096, 128000),
    ]


def draw(rng):
    op = rng.choice(("linear", "linear", "linear_grad", "gated", "gated_grad", "loss", "loss_grad"))
    type_ = rng.choice(("bf16", "bf16", "fp16", "fp32"))

    def size(lo, hi, step):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, n // step * step) if rng.random() < 0.6 else n  # whole steps, or whatever comes

    most = 1.0e12 if type_ == "fp32" else 6.0e12  # operations; the largest listed case has 12.9e12
    while True:
        N = size(1, 8192, 1)
        Cs = size(64, 9216, 64)
        Ct = size(512, 128000, 256) if op.startswith("loss") else size(64, 16384, 64)
        c = case(None, op, type_, N, Cs, Ct,
                 act="none" if op.startswith("loss") else rng.choice(ACTS[1:] if op.startswith("gated") else ACTS),
                 bias=rng.random() < 0.5, residual=op == "linear" and rng.random() < 0.5, strided=rng.random() < 0.3)
        if work(c)["flops"] <= most:
            return c


def work(c):
    s = 4 if c["type"] == "fp32" else 2
    N, Cs, Ct, op = c["N"], c["Cs"], c["Ct"], c["op"]
    x, b = N * Cs, (1 if c["bias"] else 0)
    if op == "linear":
        return {"bytes": s * (x + Ct * Cs + b * Ct + N * Ct * (2 if c["residual"] else 1)), "flops": 2 * N * Cs * Ct}
    if op == "linear_grad":
        pre = 0 if c["act"] == "none" else N * Ct
        return {"bytes": s * (N * Ct + pre + 2 * x + 2 * Ct * Cs + b * Ct), "flops": 4 * N * Cs * Ct}
    if op == "gated":
        return {"bytes": s * (x + 2 * Ct * Cs + 2 * b * Ct + N * Ct), "flops": 4 * N * Cs * Ct}
    if op == "gated_grad":
        return {"bytes": s * (3 * N * Ct + 2 * x + 4 * Ct * Cs + 2 * b * Ct), "flops": 8 * N * Cs * Ct}
    if op == "loss":
        return {"bytes": s * (x + Ct * Cs + b * Ct) + 12 * N, "flops": 2 * N * Cs * Ct}
    return {"bytes": s * (2 * x + 2 * Ct * Cs + 2 * b * Ct) + 16 * N, "flops": 6 * N * Cs * Ct}


# ------------------------------------------------------------------ inputs

def _inputs(c, seed):
    """Activations of unit size, weights of 1 / sqrt(C_s), labels with one row
    in ten left out, gradients as a mean over the rows gives them."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    T = TYPES[c["type"]]
    N, Cs, Ct, op = c["N"], c["Cs"], c["Ct"], c["op"]
    gated, loss = op.startswith("gated"), op.startswith("loss")
    rows = 2 * Ct if gated else Ct

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).to(T)

    d = {"x": normal(N, Cs + 64)[:, :Cs] if c["strided"] else normal(N, Cs),
         "w": normal(rows, Cs, scale=(2.0 if loss else 1.0) / math.sqrt(Cs)),
         "bias": normal(rows, scale=0.3) if c["bias"] else None}
    if c["residual"]:
        d["residual"] = normal(N, Ct)
    if loss:
        labels = torch.randint(0, Ct, (N,), generator=g, device=DEV)
        out = torch.rand((N,), generator=g, device=DEV) < 0.1
        out[0] = False
        d["labels"] = torch.where(out, torch.full_like(labels, -100), labels)
        d["dloss"] = torch.full((N,), 1.0, device=DEV) / (~out).sum()
    if op in ("linear_grad", "gated_grad"):
        d["dy"] = normal(N, Ct, scale=1.0 / math.sqrt(N))
        d["pre"] = None
        if c["act"] != "none":  # what the forward pass kept
            z = d["x"].float() @ d["w"].float().t()
            d["pre"] = (z if d["bias"] is None else z + d["bias"].float()).to(T)
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    torch.cuda.synchronize()
    return {"case": case, **d}


# -------------------------------------------------------------- plain form

def _act(z, act):
    if act == "relu":
        return z * (z > 0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _product(x, w, bias):
    z = x.float() @ w.float().t()
    return z if bias is None else z + bias.float()


def _gradients(dz, x, w, bias):
    T = x.dtype
    dx, dw = dz @ w.float(), dz.t() @ x.float()
    return {"dx": dx.to(T), "dw": dw.to(T), **({} if bias is None else {"dbias": dz.sum(0).to(T)})}


def _plain(s):
    c, x, w, bias = s["case"], s["x"], s["w"], s["bias"]
    op, act, T, Ct = c["op"], c["act"], x.dtype, c["Ct"]
    if op == "linear":
        y = _act(_product(x, w, bias), act)
        return (y + s["residual"].float() if c["residual"] else y).to(T)
    if op == "linear_grad":
        dy = s["dy"].float()
        return _gradients(dy if act == "none" else dy * _slope(s["pre"].float(), act), x, w, bias)
    if op == "gated":
        z = _product(x, w, bias)
        return (_act(z[:, :Ct], act) * z[:, Ct:]).to(T)
    if op == "gated_grad":
        dy, g, u = s["dy"].float(), s["pre"][:, :Ct].float(), s["pre"][:, Ct:].float()
        return _gradients(torch.cat([dy * u * _slope(g, act), dy * _act(g, act)], 1), x, w, bias)
    z = _product(x, w, bias)
    top = z.max(1, keepdim=True).values
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    counted = s["labels"] >= 0
    label = torch.where(counted, s["labels"], torch.zeros_like(s["labels"]))[:, None]
    loss = torch.where(counted, (lse - z.gather(1, label))[:, 0], torch.zeros_like(lse[:, 0]))
    if op == "loss":
        return loss
    d = torch.exp(z - lse)
    d.scatter_add_(1, label, torch.full_like(lse, -1.0))
    d *= torch.where(counted, s["dloss"], torch.zeros_like(s["dloss"]))[:, None]
    return {"loss": loss, **_gradients(d, x, w, bias)}


# ------------------------------------------------------------ this package

def _own(s):
    from paper_1512_06473_amd import api
    c, x, w, bias = s["case"], s["x"], s["w"], s["bias"]
    op, act = c["op"], c["act"]
    if op == "linear":
        return api.linear_forward(x, w, bias, act=act, residual=s.get("residual"))
    if op == "gated":
        return api.gated_forward(x, w, bias, act=act)
    if op == "loss":
        return api.linear_xent_forward(x, w, s["labels"], bias)[0]
    if op == "linear_grad":
        dx, dw, db = api.linear_backward(s["dy"], x, w, act=act, pre=s["pre"], need_dbias=bias is not None)
        out = {}
    elif op == "gated_grad":
        dx, dw, db = api.gated_backward(s["dy"], x, w, s["pre"], act=act, need_dbias=bias is not None)
        out = {}
    else:
        loss, lse = api.linear_xent_forward(x, w, s["labels"], bias)
        dx, dw, db = api.linear_xent_backward(s["dloss"], lse, x, w, s["labels"], bias)
        out = {"loss": loss}
    return {**out, "dx": dx, "dw": dw, **({} if bias is None else {"dbias": db})}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------- exact

def exact(case, seed):
    """From the definitions, in float64, a block of rows at a time."""
    d = _inputs(case, seed)
    op, act, Ct = case["op"], case["act"], case["Ct"]
    x, w = d["x"].double(), d["w"].double()
    b = None if d["bias"] is None else d["bias"].double()
    phi = torch.distributions.Normal(0.0, 1.0)

    def value(z):
        if act == "relu":
            return z.clamp(min=0)
        if act == "gelu":
            return z * phi.cdf(z)
        if act == "gelu_tanh":
            return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return z * torch.sigmoid(z) if act == "silu" else z

    def slope(z):
        with torch.enable_grad():
            z = z.detach().requires_grad_(True)
            return torch.autograd.grad(value(z).sum(), z)[0]

    dz_all, outs, losses = [], [], []
    for r in range(0, case["N"], 1024):
        rows = slice(r, min(r + 1024, case["N"]))
        if op.endswith("grad") and not op.startswith("loss"):
            dy = d["dy"][rows].double()
            pre = None if d["pre"] is None else d["pre"][rows].double()
            if op == "linear_grad":
                dz_all.append(dy if pre is None else dy * slope(pre))
            else:
                g, u = pre[:, :Ct], pre[:, Ct:]
                dz_all.append(torch.cat([dy * u * slope(g), dy * value(g)], 1))
            continue
        z = torch.mm(x[rows], w.t())
        if b is not None:
            z += b
        if op == "linear":
            y = value(z)
            outs.append(y + d["residual"][rows].double() if case["residual"] else y)
        elif op == "gated":
            outs.append(value(z[:, :Ct]) * z[:, Ct:])
        else:
            lp = torch.log_softmax(z, 1)
            lab = d["labels"][rows]
            on = (lab >= 0).nonzero()[:, 0]
            loss = torch.zeros(lab.shape[0], dtype=torch.float64, device=DEV)
            loss[on] = -lp[on, lab[on]]
            losses.append(loss)
            if op == "loss_grad":
                p = lp.exp()
                p[on, lab[on]] -= 1.0
                weight = torch.zeros_like(loss)
                weight[on] = d["dloss"][rows].double()[on]
                dz_all.append(p * weight[:, None])
    if outs:
        return torch.cat(outs)
    if op == "loss":
        return torch.cat(losses)
    dx, dw, db = [], torch.zeros_like(w), torch.zeros(w.shape[0], dtype=torch.float64, device=DEV)
    for k, r in enumerate(range(0, case["N"], 1024)):
        dz = dz_all[k]
        dx.append(torch.mm(dz, w))
        dw += torch.mm(dz.t(), x[r:r + 1024])
        db += dz.sum(0)
    return {**({"loss": torch.cat(losses)} if losses else {}), "dx": torch.cat(dx), "dw": dw,
            **({} if b is None else {"dbias": db})}
