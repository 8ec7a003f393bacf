"""Refusals of the operators on caller-owned arrays, through the C ABI without a GPU: every bad argument is turned
into a status before anything is queued (the pointers below are never followed), and what the workspaces need."""
import ctypes as C

import pytest

P = 1 << 20   # an address that is aligned to everything and never read


@pytest.fixture(scope="module")
def L():
    import paper_1810_08313_amd as p
    return p.lib()


def R(p=P, row=64, replica=0):
    from paper_1810_08313_amd.binding import LcRows
    return LcRows(p, row, replica)


def test_layer_norm_refuses(L):
    def fwd(m=2, rows=4, cols=64, dtype=0, x=R(replica=256), gain=P, bias=P, rep=64, eps=1e-5, y=R(replica=256), stats=P):
        return L.lc_layer_norm(m, rows, cols, dtype, x, gain, bias, rep, eps, y, stats, None)
    assert fwd(rows=0) == 0                                   # nothing to do
    assert fwd(m=0) == -1 and fwd(m=65536) == -1 and fwd(rows=-1) == -1 and fwd(cols=0) == -1
    assert fwd(dtype=2) == -1 and fwd(eps=-1.0) == -1 and fwd(eps=float("nan")) == -1 and fwd(rep=-1) == -1
    assert fwd(x=R(None)) == -1 and fwd(y=R(None)) == -1
    assert fwd(x=R(row=63)) == -1 and fwd(x=R(replica=-64)) == -1
    assert fwd(y=R(replica=255)) == -1 and fwd(y=R(replica=0)) == -1   # two replicas in one place
    assert fwd(x=R(P + 2)) == -4 and fwd(x=R(P + 1), dtype=1) == -4 and fwd(gain=P + 1) == -4 and fwd(stats=P + 2) == -4

    def bwd(m=2, rows=4, cols=64, dtype=0, x=R(replica=256), dy=R(replica=256), gain=P, stats=P, dx=R(replica=256), dg=P, db=P,
            rep=64, ws=P, n=1 << 20):
        return L.lc_layer_norm_grad(m, rows, cols, dtype, x, dy, gain, 64, stats, dx, dg, db, rep, ws, n, None)
    need = L.lc_layer_norm_workspace_bytes(2, 4, 64)
    assert need >= 2 * 2 * 64 * 4 and L.lc_layer_norm_workspace_bytes(0, 4, 64) == 0
    assert bwd(m=0) == -1 and bwd(dtype=-1) == -1 and bwd(stats=None) == -1 and bwd(rep=63) == -1 and bwd(dy=R(row=1)) == -1
    assert bwd(n=need - 1) == -5 and bwd(ws=None) == -5 and bwd(ws=P + 128) == -4 and bwd(dx=R(replica=0)) == -1
    assert bwd(rows=-1) == -1 and bwd(db=P + 2) == -4


def head_args(**kw):
    from paper_1810_08313_amd.binding import LcHeadArgs
    h = LcHeadArgs(m=2, inputs=64, rows=8, classes=1000, dtype=1, grad_dtype=1, A=R(row=64, replica=512), W=R(row=1000, replica=64000),
                   bias=P, bias_replica=1000, labels=P, label_replica=8, loss=P, row_loss=P, row_loss_replica=8,
                   dA=R(2 * P, row=64, replica=512), dW=R(3 * P, row=1000, replica=64000), db=P, db_replica=1000)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


BAD_HEADS = [
    (dict(m=0), -1), (dict(rows=-1), -1), (dict(inputs=0), -1), (dict(classes=0), -1), (dict(dtype=2), -1),
    (dict(A=R(None)), -1), (dict(W=R(None)), -1), (dict(labels=None), -1), (dict(loss=None), -1), (dict(A=R(row=63)), -1),
    (dict(W=R(row=999)), -1), (dict(bias_replica=-1), -1), (dict(row_loss_replica=7), -1), (dict(A=R(P + 1)), -4),
    (dict(labels=P + 2), -4), (dict(bias=P + 2), -4), (dict(rows=1 << 25), -8), (dict(classes=(1 << 22) + 1, W=R(row=1 << 23)), -8),
    (dict(inputs=(1 << 20) + 1), -8),
]
BAD_GRADS = [
    (dict(dA=R(row=64, replica=512)), -1), (dict(dW=R(row=1000, replica=64000)), -1),   # where A and W stand
    (dict(grad_dtype=3), -1), (dict(dA=R(None)), -1), (dict(dW=R(None)), -1), (dict(dA=R(2 * P, row=64, replica=0)), -1),
    (dict(dW=R(row=1000, replica=0)), -1), (dict(db_replica=999), -1), (dict(db=P + 1), -4),
]


def test_softmax_head_refuses(L):
    for kw, want in BAD_HEADS + BAD_GRADS:
        h = head_args(**kw)
        grad_only = (kw, want) in BAD_GRADS
        assert L.lc_softmax_head_grad(C.byref(h), P, 1 << 40, None) == want, kw
        assert L.lc_softmax_head_workspace_bytes(C.byref(h), 1) == 0, kw
        assert (L.lc_softmax_head_workspace_bytes(C.byref(h), 0) > 0) == grad_only, kw
        if not grad_only:
            assert L.lc_softmax_head_loss(C.byref(h), P, 1 << 40, None) == want, kw
    h = head_args()
    for fn, grad in ((L.lc_softmax_head_loss, 0), (L.lc_softmax_head_grad, 1)):
        n = L.lc_softmax_head_workspace_bytes(C.byref(h), grad)
        assert fn(None, P, n, None) == -1
        assert fn(C.byref(h), P, n - 1, None) == -5 and fn(C.byref(h), None, n, None) == -5
        assert fn(C.byref(h), P + 64, n, None) == -4
    assert L.lc_softmax_head_workspace_bytes(None, 0) == 0


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,d,classes", [(8192, 2048, 128000), (1 << 20, 64, 300), (1, 4096, 1 << 22), (100000, 512, 50257)])
def test_softmax_head_workspace_stays_bounded(L, rows, d, classes, dtype):
    """A whole batch's logits are never kept: beyond what a chunk of rows needs there are only copies of the operands."""
    e = 2 if dtype else 4
    h = head_args(m=1, rows=rows, inputs=d, classes=classes, dtype=dtype, grad_dtype=dtype, A=R(row=d), W=R(row=classes),
                  dA=R(2 * P, row=d), dW=R(3 * P, row=classes), db=P)
    n = L.lc_softmax_head_workspace_bytes(C.byref(h), 1)
    chunk = min(rows + 64, 65536)
    kept = max(2 << 30, 256 * (classes + 64) * 10) * 1.1
    copies = chunk * (d + 64) * (4 * e + 8) + 3 * d * (classes + 64) * 4 + rows * 12 + (2 * classes * (chunk // 64 + 2)) * 4
    shares = 256 * 256 * 256 * 4 * 2
    assert 0 < n < kept + copies + shares, (n, kept, copies)


def test_orthogonal_refuses(L):
    def orth(m=2, rows=8, cols=64, dtype=0, src=R(replica=512), dst=R(replica=512), steps=5, ws=P, n=1 << 30):
        return L.lc_orthogonalize(m, rows, cols, dtype, src, dst, steps, ws, n, None)
    need = L.lc_orthogonal_workspace_bytes(2, 8, 64, 0)
    assert need > 0 and L.lc_orthogonal_workspace_bytes(2, 8, 64, 2) == 0 and L.lc_orthogonal_workspace_bytes(2, 0, 64, 0) == 0
    assert orth(m=0) == -1 and orth(rows=0) == -1 and orth(cols=32769) == -1 and orth(dtype=2) == -1
    assert orth(steps=0) == -1 and orth(steps=17) == -1 and orth(src=R(None)) == -1 and orth(dst=R(replica=0)) == -1
    assert orth(src=R(P + 2)) == -4 and orth(n=need - 1) == -5 and orth(ws=None) == -5 and orth(ws=P + 16) == -4

    def upd(X=R(P, replica=512), V=R(2 * P, replica=512), G=R(3 * P, replica=512), lr=0.1, beta=0.9, wd=0.0, steps=5, ws=4 * P, n=1 << 30):
        return L.lc_update_orthogonal(2, 8, 64, X, V, G, lr, beta, wd, steps, ws, n, None)
    assert upd(lr=0.0) == -1 and upd(beta=1.0) == -1 and upd(beta=-0.1) == -1 and upd(wd=-1.0) == -1 and upd(lr=float("nan")) == -1
    assert upd(V=R(P, replica=512)) == -1 and upd(G=R(2 * P, replica=512)) == -1 and upd(X=R(replica=0)) == -1 and upd(steps=0) == -1
    assert upd(n=need - 1) == -5


def test_update_from_grad_orthogonal_refuses(L):
    import paper_1810_08313_amd as pkg
    assert L.lc_update_from_grad_orthogonal(None, 5, P, 1 << 30) == -1 and L.lc_update_orthogonal_bytes(None) == 0
    for kind, dims, want in ((pkg.KIND_MLP, [8, 4, 3], True), (pkg.KIND_QUAD, [64], False)):
        md = pkg.make_model(kind, dims, B=4, N=10, E=10)
        h = C.c_void_p()
        assert L.lc_init(2, pkg.lc_param_count(md), C.byref(md), 1, C.byref(h)) == 0
        assert (L.lc_update_orthogonal_bytes(h) > 0) == want
        assert L.lc_update_from_grad_orthogonal(h, 5, P, 1 << 30) == -3      # not attached
        assert L.lc_update_from_grad_orthogonal(h, 0, P, 1 << 30) == -1
        L.lc_destroy(h)


def test_bindings_refuse_host_tensors():
    torch = pytest.importorskip("torch")
    import paper_1810_08313_amd as pkg
    x = torch.zeros(2, 3, 8)
    with pytest.raises(pkg.LcError):
        pkg.layer_norm(x)
    with pytest.raises(pkg.LcError):
        pkg.orthogonalize(x)
    with pytest.raises(pkg.LcError):
        pkg.softmax_head_loss(x, torch.zeros(2, 8, 5), None, torch.zeros(2, 3, dtype=torch.int32))
