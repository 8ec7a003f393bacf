"""Operators of larger models on the stack of replicas, as cases that can be timed and compared.

Every array has the replicas as its first axis, as the rows of X have them. Three operators, each with
what a training step needs of it:

  norm       layer normalisation of the last axis with a gain and a bias per replica; "grad": its backward
             pass, the reduction of the gain's and the bias's gradient over the rows included
  head       softmax cross-entropy over many classes from the last hidden layer, Z = A W + b, with W as it
             stands in a row of X, [d, classes]; rows whose label is negative are left out, the loss is the
             mean over the others; "grad": dA, dW and db of that mean as well
  orth       the matrix that Newton-Schulz products make of a gradient, Q X with singular values near 1;
             "update": the momentum step of one weight matrix that takes it as its direction

The plain forms below are elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"

# X <- a X + b (X X^T) X + c (X X^T)^2 X, five times from X / |X|_F: every singular value in (0, 1] ends near 1
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315
STEPS = 5


# ------------------------------------------------------------------------------------- the cases

def _norm(name, m, rows, cols, bf16, grad):
    return dict(name=name, op="norm", m=m, rows=rows, cols=cols, bf16=bf16, grad=grad)


def _head(name, m, rows, d, classes, bf16, grad, left_out):
    return dict(name=name, op="head", m=m, rows=rows, d=d, classes=classes, bf16=bf16, grad=grad, left_out=left_out)


def _orth(name, m, rows, cols, bf16, update):
    return dict(name=name, op="orth", m=m, rows=rows, cols=cols, bf16=bf16, update=update)


def listed():
    return [
        # one mini-batch of a small network on four workers: nothing but launch latency
        _norm("norm_one_batch", 4, 32, 256, False, False),
        # the rows of a long batch of sequences: as fast as memory
        _norm("norm_long", 2, 8192, 4096, True, False),
        # sixteen workers of 100 samples at a width that is no power of two: many replicas, few rows each
        _norm("norm_grad_ragged", 16, 100, 1500, False, True),
        # the backward pass of a long batch, a row short of a round number
        _norm("norm_grad_long", 4, 8191, 2048, True, True),
        # the loss of a single token: the weights are read once and little else happens
        _head("head_loss_one_token", 1, 1, 2048, 32000, True, False, 0),
        # a thousand classes behind a small hidden layer, mini-batches of 64: fp32 masters as they stand in X
        _head("head_grad_small", 8, 64, 256, 1000, False, True, 0),
        # an odd vocabulary, eight workers, a quarter of each batch is padding
        _head("head_grad_odd", 8, 128, 512, 50257, True, True, 32),
        # a long batch against a large vocabulary: matrix products of the largest kind
        _head("head_grad_long", 1, 8192, 2048, 128000, True, True, 100),
        # the gradients of one small layer on eight workers, wider than high and no size round
        _orth("orth_small", 8, 300, 784, False, False),
        # one large square matrix in bf16
        _orth("orth_square", 1, 4096, 4096, True, False),
        # the momentum step of a hidden layer on sixteen workers
        _orth("update_hidden", 16, 1024, 1024, False, True),
        # the same of an odd layer that is higher than wide
        _orth("update_tall", 3, 1301, 500, False, True),
    ]


def _log(rng, lo, hi):
    """A whole number, its logarithm uniform."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "head", "head", "orth", "orth"])
    bf16, half = rng.random() < 0.5, rng.random() < 0.5
    while True:
        m = _log(rng, 1, 16)
        if op == "norm":
            c = _norm("", m, _log(rng, 1, 16384), _log(rng, 8, 8192), bf16, half)
            if m * c["rows"] * c["cols"] > 4 * 8191 * 2048:
                continue
        elif op == "head":
            rows = _log(rng, 1, 8192)
            c = _head("", m, rows, _log(rng, 32, 4096), _log(rng, 300, 128000), bf16, half,
                      int(rows * rng.choice([0, 0, 0.1, 0.4])))
            # fp32 operands cost several times the products of bf16
            most = 8192 * 2048 * 128000 // (1 if bf16 else 16)
            if m * rows * c["d"] * c["classes"] > most or m * c["d"] * c["classes"] > 1 << 28 or \
                    m * rows * c["classes"] > 1 << 29:
                continue
        else:
            c = _orth("", m, _log(rng, 24, 4096), _log(rng, 24, 4096), bf16 and half, not half)
            small = min(c["rows"], c["cols"])
            if m * small * c["rows"] * c["cols"] > 4096 ** 3 // (1 if c["bf16"] else 4):
                continue
        del c["name"]
        return c


# ------------------------------------------------------------------------------------- the inputs

def _normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = torch.bfloat16 if case["bf16"] else torch.float32
    m, s = case["m"], {"case": case}
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # activations with an offset and a spread of their own in every row
        s["x"] = (_normal(g, m, rows, cols) * (0.5 + 2 * torch.rand(m, rows, 1, device=DEV, generator=g))
                  + 0.3 * _normal(g, m, rows, 1)).to(t)
        s["gain"] = 1 + 0.1 * _normal(g, m, cols)
        s["bias"] = 0.1 * _normal(g, m, cols)
        s["eps"] = 1e-5
        if case["grad"]:
            s["dy"] = (_normal(g, m, rows, cols) * 1e-3).to(t)
            x = s["x"].double()
            mean = x.mean(-1)
            s["stats"] = torch.stack([mean, (x.var(-1, unbiased=False) + s["eps"]).rsqrt()], -1).float()
    elif case["op"] == "head":
        rows, d, classes = case["rows"], case["d"], case["classes"]
        s["A"] = _normal(g, m, rows, d).to(t)                                  # normalised activations
        s["W"] = (_normal(g, m, d, classes) * (1.5 / math.sqrt(d))).to(t)      # logits spread by 1.5
        s["b"] = 0.1 * _normal(g, m, classes)
        # few classes are frequent, most are rare
        lab = (torch.rand(m, rows, device=DEV, generator=g) ** 3 * classes).to(torch.int32).clamp_(max=classes - 1)
        if case["left_out"]:
            order = torch.rand(m, rows, device=DEV, generator=g).argsort(1)
            lab[order < case["left_out"]] = -1
        s["labels"] = lab
    else:
        rows, cols = case["rows"], case["cols"]
        # a gradient as activations times deltas of a batch, its directions of unequal weight, and noise over it
        k = max(1, min(128, rows, cols))
        u = _normal(g, m, rows, k) * torch.linspace(1, 0.05, k, device=DEV)
        s["G"] = ((u @ _normal(g, m, k, cols)) / math.sqrt(k) + 0.02 * _normal(g, m, rows, cols)).mul_(1e-2).to(t)
        if case["update"]:
            s["X"] = _normal(g, m, rows, cols) * math.sqrt(2 / rows)
            s["V"] = (u @ _normal(g, m, k, cols)) / math.sqrt(k) * 3e-2 + 1e-3 * _normal(g, m, rows, cols)
            s["lr"], s["beta"], s["wd"] = 0.02, 0.9, 1e-3
    return s


# ------------------------------------------------------------------------------------- one pass

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_1810_08313_amd as pkg
    c = s["case"]
    if c["op"] == "norm":
        if not c["grad"]:
            return pkg.layer_norm(s["x"], s["gain"], s["bias"], s["eps"])
        return pkg.layer_norm_grad(s["x"], s["dy"], s["gain"], s["stats"])
    if c["op"] == "head":
        if not c["grad"]:
            return pkg.softmax_head_loss(s["A"], s["W"], s["b"], s["labels"])
        return pkg.softmax_head_grad(s["A"], s["W"], s["b"], s["labels"])
    if not c["update"]:
        return pkg.orthogonalize(s["G"], STEPS)
    pkg.update_orthogonal(s["X"], s["V"], s["G"], s["lr"], s["beta"], s["wd"], STEPS)
    return s["X"], s["V"]


def _plain(s):
    c = s["case"]
    if c["op"] == "norm":
        return _plain_norm_grad(s) if c["grad"] else _plain_norm(s)
    if c["op"] == "head":
        return _plain_head(s)
    if not c["update"]:
        return _plain_orth(s["G"].float()).to(s["G"].dtype)
    rows, cols = c["rows"], c["cols"]
    s["V"].mul_(s["beta"]).add_(s["G"])
    step = math.sqrt(max(1.0, cols / rows)) * _plain_orth(s["V"]) + s["wd"] * s["X"]
    s["X"].sub_(s["lr"] * step)
    return s["X"], s["V"]


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    r = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + s["eps"])
    y = d * r * s["gain"][:, None] + s["bias"][:, None]
    return y.to(s["x"].dtype), torch.cat([mean, r], -1)


def _plain_norm_grad(s):
    x, dy = s["x"].float(), s["dy"].float()
    mean, r = s["stats"][..., :1], s["stats"][..., 1:]
    n = (x - mean) * r
    h = dy * s["gain"][:, None]
    dx = r * (h - h.mean(-1, keepdim=True) - n * (h * n).mean(-1, keepdim=True))
    return dx.to(s["x"].dtype), (dy * n).sum(1), dy.sum(1)


def _plain_head(s):
    A, W, lab = s["A"].float(), s["W"].float(), s["labels"].long()
    keep = lab >= 0
    at = lab.clamp(min=0)[..., None]
    n = keep.sum(1).clamp(min=1).float()
    A = torch.where(keep[..., None], A, 0.0)
    z = A @ W + s["b"][:, None]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    sums = e.sum(-1, keepdim=True)
    row = torch.where(keep, (top + torch.log(sums) - z.gather(-1, at))[..., 0], 0.0)
    loss = row.sum(1) / n
    if not s["case"]["grad"]:
        return loss, row
    dz = (e / sums).scatter_add_(-1, at, torch.full_like(sums, -1.0))
    dz *= (keep / n[:, None])[..., None]
    t = s["A"].dtype
    return loss, (dz @ W.transpose(1, 2)).to(t), (A.transpose(1, 2) @ dz).to(t), dz.sum(1).to(t)


def _plain_orth(M):
    x = M if M.shape[1] <= M.shape[2] else M.transpose(1, 2)
    x = x / torch.sqrt((x * x).sum((1, 2), keepdim=True))
    for _ in range(STEPS):
        a = x @ x.transpose(1, 2)
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    return x if M.shape[1] <= M.shape[2] else x.transpose(1, 2)


# ------------------------------------------------------------------------------------- what it cannot do without

def work(case):
    e = 2 if case["bf16"] else 4
    m = case["m"]
    if case["op"] == "norm":
        n, p, rows = m * case["rows"] * case["cols"], m * case["cols"] * 4, m * case["rows"] * 8
        if case["grad"]:
            return {"bytes": 3 * n * e + 3 * p + rows, "flops": 14 * n}
        return {"bytes": 2 * n * e + 2 * p + rows, "flops": 8 * n}
    if case["op"] == "head":
        rows = m * (case["rows"] - case["left_out"])
        a, w, c = m * case["rows"] * case["d"] * e, m * case["d"] * case["classes"] * e, m * case["classes"]
        flops = 2 * rows * case["d"] * case["classes"]
        if case["grad"]:
            return {"bytes": 2 * a + 2 * w + c * (4 + e) + m * case["rows"] * 4, "flops": 3 * flops}
        return {"bytes": a + w + 4 * c + m * case["rows"] * 8, "flops": flops}
    small, n = min(case["rows"], case["cols"]), m * case["rows"] * case["cols"]
    # X X^T and its square are symmetric: half of either
    flops = STEPS * small * (3 * n + m * small * small)
    return {"bytes": n * 20 if case["update"] else 2 * n * e, "flops": flops}


# ------------------------------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    if case["op"] == "norm":
        x, gain = s["x"].to(f8), s["gain"].to(f8).unsqueeze(1)
        if not case["grad"]:
            var, mean = torch.var_mean(x, -1, correction=0)
            r = (var + s["eps"]) ** -0.5
            y = (x - mean.unsqueeze(-1)) * r.unsqueeze(-1)
            return y * gain + s["bias"].to(f8).unsqueeze(1), torch.stack((mean, r), -1)
        dy, st = s["dy"].to(f8), s["stats"].to(f8)
        n = (x - st[..., 0:1]) * st[..., 1:2]
        dgain, dbias = torch.einsum("mrc,mrc->mc", dy, n), dy.sum(1)
        dy *= gain
        proj = torch.einsum("mrc,mrc->mr", dy, n) / case["cols"]
        dx = (dy - dy.mean(-1, keepdim=True) - proj.unsqueeze(-1) * n) * st[..., 1:2]
        return dx, dgain, dbias
    if case["op"] == "head":
        m, rows = case["m"], case["rows"]
        loss, each = torch.zeros(m, dtype=f8, device=DEV), torch.zeros(m, rows, dtype=f8, device=DEV)
        dA = torch.zeros(m, rows, case["d"], dtype=f8, device=DEV)
        dW, db = [], []
        for i in range(m):
            W = s["W"][i].to(f8)
            gw, gb = torch.zeros_like(W), torch.zeros(case["classes"], dtype=f8, device=DEV)
            kept = torch.nonzero(s["labels"][i] >= 0).flatten()
            for part in kept.split(1024):
                a, y = s["A"][i, part].to(f8), s["labels"][i, part].long()
                z = torch.addmm(s["b"][i].to(f8), a, W)
                lse = torch.logsumexp(z, 1)
                pick = torch.arange(len(part), device=DEV)
                each[i, part] = lse - z[pick, y]
                if case["grad"]:
                    z = torch.softmax(z, 1)
                    z[pick, y] -= 1
                    z /= len(kept)
                    dA[i, part] = z @ W.T
                    gw += a.T @ z
                    gb += z.sum(0)
            loss[i] = each[i].sum() / max(1, len(kept))
            if case["grad"]:
                dW.append(gw)
                db.append(gb)
        return (loss, dA, torch.stack(dW), torch.stack(db)) if case["grad"] else (loss, each)
    if case["update"]:
        v = s["beta"] * s["V"].to(f8) + s["G"].to(f8)
        x = s["X"].to(f8)
        scale = max(1.0, case["cols"] / case["rows"]) ** 0.5
        return x - s["lr"] * (scale * _exact_orth(v) + s["wd"] * x), v
    return _exact_orth(s["G"].to(f8))


def _exact_orth(v):
    """The same polynomial of the singular values, each product on the smaller side."""
    x = v / torch.linalg.vector_norm(v, dim=(1, 2), keepdim=True)
    tall = v.shape[1] > v.shape[2]
    eye = torch.eye(min(v.shape[1:]), dtype=v.dtype, device=v.device)
    for _ in range(STEPS):
        gram = torch.bmm(x.mT.contiguous(), x) if tall else torch.bmm(x, x.mT.contiguous())
        p = NS_A * eye + torch.bmm(gram, NS_B * eye + NS_C * gram)
        x = torch.bmm(x, p) if tall else torch.bmm(p, x)
    return x
