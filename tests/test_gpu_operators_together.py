"""The operators as a training step uses them: rows of X hold a layer norm's gain and bias, a hidden layer and a head over
many classes; the gradients of all of them go into rows of G by hand, and the update and the averaging step follow.
Everything is followed in 64 bits next to it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1810_08313_amd as p
    p.lib()
    return p


class _Net:
    """x -> layer norm -> W1 -> + x -> layer norm -> head, fp32; parameters in rows [gain1 bias1 W1 gain2 bias2 W b]."""

    def __init__(self, m, d, classes):
        self.m, self.d, self.C = m, d, classes
        sizes = [("g1", (d,)), ("b1", (d,)), ("W1", (d, d)), ("g2", (d,)), ("b2", (d,)), ("W", (d, classes)), ("b", (classes,))]
        self.at, off = {}, 0
        for k, s in sizes:
            self.at[k] = (off, s)
            off += int(np.prod(s))
        self.P = off

    def view(self, T, k):
        off, s = self.at[k]
        st = (T.stride(0), s[1], 1) if len(s) == 2 else (T.stride(0), 1)
        return T.as_strided((self.m, *s), st, T.storage_offset() + off)

    def start(self, seed):
        import torch
        import paper_1810_08313_amd as pkg
        X = torch.zeros(self.m, pkg.lc_row_stride(self.P), device="cuda")
        g = torch.Generator(device="cuda").manual_seed(seed)
        for k in ("g1", "g2"):
            self.view(X, k).fill_(1.0)
        for k in ("W1", "W"):
            w = self.view(X, k)
            w.copy_((torch.randn(w.shape[1:], device="cuda", generator=g) / self.d ** 0.5).expand(w.shape))
        return X


def _step(pkg, net, X, G, x, y):
    """Loss [m] of a batch x [m, rows, d] and all gradients into G."""
    import torch
    P, Q = (lambda k: net.view(X, k)), (lambda k: net.view(G, k))
    n1, s1 = pkg.layer_norm(x, P("g1"), P("b1"))
    h = x + torch.stack([n1[i] @ P("W1")[i] for i in range(net.m)])
    n2, s2 = pkg.layer_norm(h, P("g2"), P("b2"))
    loss, dn2, _, _ = pkg.softmax_head_grad(n2, P("W"), P("b"), y, dW=Q("W"), db=Q("b"))
    dh, _, _ = pkg.layer_norm_grad(h, dn2, P("g2"), s2, dgain=Q("g2"), dbias=Q("b2"))
    dn1 = torch.empty_like(n1)
    for i in range(net.m):
        Q("W1")[i].copy_(n1[i].T @ dh[i])
        dn1[i] = dh[i] @ P("W1")[i].T
    pkg.layer_norm_grad(x, dn1, P("g1"), s1, dgain=Q("g1"), dbias=Q("b1"))
    return loss


def _reference(net, X, x, y):
    """The same loss and gradient in 64 bits by differentiation, on the CPU."""
    import torch
    X = X.detach().double().cpu().requires_grad_(True)
    x, y = x.double().cpu(), y.cpu().long()
    losses = []
    P = lambda k: net.view(X, k)  # noqa: E731

    def norm(v, g, b):
        mean = v.mean(-1, keepdim=True)
        return (v - mean) / ((v - mean).pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * g + b
    for i in range(net.m):
        h = x[i] + norm(x[i], P("g1")[i], P("b1")[i]) @ P("W1")[i]
        z = norm(h, P("g2")[i], P("b2")[i]) @ P("W")[i] + P("b")[i]
        keep = y[i] >= 0
        losses.append((torch.logsumexp(z, -1)[keep] - z[keep].gather(1, y[i][keep][:, None])[:, 0]).mean())
    sum(losses).backward()
    return torch.stack(losses).detach(), X.grad


def _batch(net, rows, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(net.m, rows, net.d, device="cuda", generator=g)
    y = torch.randint(0, net.C, (net.m, rows), device="cuda", generator=g, dtype=torch.int32)
    y[:, rows - 5:] = -1                       # padding
    return x, y


def test_a_step_of_every_replica(pkg):
    import torch
    net = _Net(3, 72, 1003)
    X = net.start(1)
    G = torch.zeros_like(X)
    x, y = _batch(net, 50, 2)
    loss = _step(pkg, net, X, G, x, y)
    torch.cuda.synchronize()
    want, grad = _reference(net, X, x, y)
    # sums of up to 1003 terms in 32 bits, four products deep: 4 * 1003 * 2^-24 = 2.4e-4 of the largest at the worst
    assert float((loss.cpu().double() - want).abs().max()) < 2.4e-4 * float(want.max())
    for k in net.at:
        a, b = net.view(G, k).cpu().double(), net.view(grad, k)
        assert float((a - b).abs().max()) <= 2.4e-4 * float(b.abs().max()), k
    assert not G[:, net.P:].any()


def test_training_with_averaging(pkg):
    """Local steps along G (the head's and the hidden layer's matrices orthogonalised, the rest by the handle's update) and an
    averaging step, twice, against the same in 64 bits."""
    import torch
    net = _Net(2, 40, 310)
    run = pkg.LocalSGD(net.m, pkg.make_model(pkg.KIND_QUAD, [net.P], lr=0.05, beta=0.9), 0,
                       qa=np.ones((net.m, net.P), np.float32), qc=np.zeros((net.m, net.P), np.float32))
    run.X.copy_(net.start(4))
    V2 = torch.zeros_like(run.X)               # momentum of the two matrices
    G = torch.zeros_like(run.X)
    Xr = run.X.double().cpu()
    Vr, Or = torch.zeros_like(Xr), torch.zeros_like(Xr)

    def orth(v):
        u, s, vt = torch.linalg.svd(v / v.norm(), full_matrices=False)
        for _ in range(5):
            s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
        return (u * s) @ vt
    for it in range(4):
        x, y = _batch(net, 30, 10 + it)
        _step(pkg, net, run.X, G, x, y)
        _, grad = _reference(net, run.X, x, y)  # the gradient at the GPU's own model: no drift to allow for
        for k in ("W1", "W"):
            pkg.update_orthogonal(net.view(run.X, k), net.view(V2, k), net.view(G, k), 0.05, 0.9)
            net.view(G, k).zero_()
        run.set_grad(G)
        run.update_from_grad()
        torch.cuda.synchronize()
        for k in net.at:
            g, xr, vr, o = (net.view(t, k) for t in (grad, Xr, Vr, Or))
            if k in ("W1", "W"):
                o.mul_(0.9).add_(g)
                for i in range(net.m):
                    a, b = xr[i].shape
                    xr[i] -= 0.05 * max(1.0, b / a) ** 0.5 * orth(o[i])
            else:
                vr.mul_(0.9).add_(g)
                xr -= 0.05 * vr
        if it % 2:
            run.average()
            Xr[:] = Xr.mean(0, keepdim=True)
            torch.cuda.synchronize()
            assert torch.equal(run.X[0], run.X[1])
        # a direction: gradients agree to 1e-4 and the smallest singular values of four samples' momentum are blown up by at
        # most 3.4445^5 = 485 relative to the largest, so that a step of 0.05 is off by less than 0.05 * 485 * 1e-4
        for k in net.at:
            a, b = net.view(run.X, k).cpu().double(), net.view(Xr, k)
            assert float((a - b).abs().max()) <= 0.05 * 485e-4 * (it + 1), (it, k)
            net.view(Xr, k).copy_(a)            # the next step starts from the same model
    assert not run.X[:, net.P:].any()
    run.close()


def test_a_step_in_a_graph(pkg):
    """The whole step captured once and replayed, with eager steps between the replays."""
    import torch
    net = _Net(2, 64, 520)
    X = net.start(6)
    G, E = torch.zeros_like(X), torch.zeros_like(X)
    x, y = _batch(net, 40, 7)

    def eager(X, G):
        P, Q = (lambda k: net.view(X, k)), (lambda k: net.view(G, k))
        n, s = pkg.layer_norm(x, P("g2"), P("b2"))
        loss, dn, _, _ = pkg.softmax_head_grad(n, P("W"), P("b"), y, dW=Q("W"), db=Q("b"))
        pkg.layer_norm_grad(x, dn, P("g2"), s, dgain=Q("g2"), dbias=Q("b2"))
        V = torch.zeros_like(P("W"))
        pkg.update_orthogonal(P("W"), V, Q("W"), 0.05, 0.0)
        return loss
    eager(X.clone(), E)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = eager(X, G)
    for k in range(3):
        X2 = X.clone()
        graph.replay()
        torch.cuda.synchronize()
        want = eager(X2, E)
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(X, X2) and torch.equal(G, E)
        x.copy_(x.flip(1))
