"""lc_softmax_head_loss and lc_softmax_head_grad against the formulas in 64 bits.

Tolerances, u = 2^-24.  A logit is a sum of d + 1 terms in 32 bits: |dz| <= (d + 8) u sum |a w|, and what is left out of
six part products of fp32 operands is below 4 u |a||w| a term; eps is the largest of a row.  Then
  loss        2 eps + (n_parts + 40) u + 4 u |loss|         (a sum of exponentials joined from parts of 256)
  p           p (2 eps + (|z - max| + 40) u)                (the argument of the exponential is rounded at its size)
  bf16        + p 2^-11 + 2^-39 (e as fp16 times 2^15), + 2^-8 |dZ| / ... rounded once: 2^-9 of a power of two, so |dZ| 2^-8
  dA, dW      sums of |dZ's error| times the other factor, (terms + 8) u of the sum of magnitudes, half a step of the
              result's type."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pkg():
    import torch
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1810_08313_amd as p
    p.lib()
    return p


def _inputs(m, rows, d, classes, bf16, seed, left_out=0.0, scale=1.5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    t = torch.bfloat16 if bf16 else torch.float32
    A, W, b = rn(m, rows, d).to(t), (rn(m, d, classes) * scale / d ** 0.5).to(t), 0.2 * rn(m, classes)
    y = torch.randint(0, classes, (m, rows), device="cuda", generator=g, dtype=torch.int32)
    y[torch.rand(m, rows, device="cuda", generator=g) < left_out] = -1
    return A, W, b, y


def _reference(A, W, b, y):
    """One replica in 64 bits: results and their bounds for fp32 and bf16 operands."""
    import torch
    bf16 = A.dtype == torch.bfloat16
    classes = W.shape[1]
    keep = (y >= 0) & (y < classes)
    a, w = A[keep].double(), W.double()
    lab, n = y[keep].long(), max(1, int(keep.sum()))
    bias = b.double() if b is not None else torch.zeros(classes, device=A.device, dtype=torch.float64)
    z = a @ w + bias
    mag = a.abs() @ w.abs() + bias.abs()
    ez = (A.shape[1] + 8 + (0 if bf16 else 4)) * U * mag
    eps = ez.max(1, keepdim=True).values if len(lab) else ez[:, :1]
    lse = torch.logsumexp(z, 1, keepdim=True)
    at = torch.arange(len(lab), device=A.device)
    row = (lse[:, 0] - z[at, lab])
    row_tol = 2 * eps[:, 0] + (classes / 256 + 40) * U + 4 * U * (row.abs() + lse[:, 0].abs())
    p = (z - lse).exp()
    ep = p * (2 * eps + ((z - lse).abs() + (lse - z.max(1, keepdim=True).values).abs() + classes / 256 + 40) * U)
    dz = p.clone()
    # the label's: minus the sum of the others
    others = (p.sum(1) - p[at, lab]).clamp(min=0) if len(lab) else p[:, 0]
    dz[at, lab] = -others
    e_label = others * (4 * eps[:, 0] + (classes / 256 + 80) * U)
    e32 = ep.clone()
    e32[at, lab] = e_label
    e = e32.clone()
    if bf16:
        e = ep + p * 2.0 ** -11 + 2.0 ** -39
        e[at, lab] = e_label
        e_db = e.clone()
        e = e + 2.0 ** -8 * (dz.abs() + e)
    else:
        e_db = e
    out = dict(loss=row.sum() / n, loss_tol=row_tol.sum() / n + 2 * U * row.abs().sum() / n, row=row, row_tol=row_tol, keep=keep,
               dA=dz @ w.T / n, dW=a.T @ dz / n, db=dz.sum(0) / n)
    terms = classes + 8
    out["dA_tol"] = (e @ w.abs().T + terms * U * (dz.abs() + e) @ w.abs().T) / n + 4 * U * out["dA"].abs()
    k = len(lab) + 8
    out["dW_tol"] = (a.abs().T @ e + k * U * (a.abs().T @ (dz.abs() + e))) / n + 4 * U * out["dW"].abs()
    out["db_tol"] = (e_db.sum(0) + k * U * (dz.abs() + e_db).sum(0)) / n + 4 * U * out["db"].abs()
    return out


def _check(name, got, want, tol, half=0.0):
    off = (got.double() - want).abs()
    tol = tol + half * (want.abs() + tol) + 1e-37
    assert bool((off <= tol).all()), (name, float((off - tol).max()), float(off.max()), float(want.abs().max()))


def _half(t):
    import torch
    return torch.finfo(torch.bfloat16).eps / 2 if t.dtype == torch.bfloat16 else 0.0


def _check_all(A, W, b, y, loss, row_loss=None, grads=None):
    import torch
    torch.cuda.synchronize()
    for i in range(A.shape[0]):
        r = _reference(A[i], W[i], b[i] if b is not None else None, y[i])
        _check("loss", loss[i], r["loss"], r["loss_tol"])
        if row_loss is not None:
            _check("rows", row_loss[i][r["keep"]], r["row"], r["row_tol"])
            assert not row_loss[i][~r["keep"]].any()
        if grads is not None:
            dA, dW, db = grads
            _check("dA", dA[i][r["keep"]], r["dA"], r["dA_tol"], _half(dA))
            assert not dA[i][~r["keep"]].any()
            _check("dW", dW[i], r["dW"], r["dW_tol"], _half(dW))
            _check("db", db[i], r["db"], r["db_tol"], _half(db))


SIZES = [   # m, rows, inputs, classes, share of rows left out
    (1, 1, 1, 1, 0), (1, 1, 8, 3, 0), (2, 3, 5, 17, 0), (2, 33, 64, 256, 0), (1, 64, 100, 257, 0), (3, 65, 33, 301, 0.2),
    (2, 128, 96, 1000, 0.5), (1, 129, 200, 515, 0), (1, 257, 130, 4099, 0.1), (2, 300, 264, 776, 0), (8, 17, 72, 2048, 0.3),
    (1, 1, 2048, 8000, 0), (1, 700, 520, 264, 0.05),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("m,rows,d,classes,left", SIZES)
def test_sizes(pkg, m, rows, d, classes, left, bf16):
    A, W, b, y = _inputs(m, rows, d, classes, bf16, rows + d + classes, left)
    print(f"softmax head m={m} rows={rows} d={d} classes={classes} bf16={bf16} left out={left}", flush=True)
    loss, row = pkg.softmax_head_loss(A, W, b, y)
    _check_all(A, W, b, y, loss, row)
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    _check_all(A, W, b, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("bf16", [False, True])
def test_gradients_of_the_other_type_and_no_bias(pkg, bf16):
    import torch
    A, W, _, y = _inputs(2, 70, 96, 520, bf16, 4, 0.1)
    other = torch.float32 if bf16 else torch.bfloat16
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, None, y, grad_dtype=other)
    assert dW.dtype == db.dtype == other and dA.dtype == A.dtype
    _check_all(A, W, None, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_left_out_touch_nothing(pkg, bf16):
    """Labels below zero and behind the last class; infinities and NaN in the activations of such rows; no row left."""
    import torch
    A, W, b, y = _inputs(3, 90, 70, 333, bf16, 6)
    y[0, ::3] = -7
    y[0, 1::3] = 333
    y[1, :] = -1
    y[2, 40:] = 2 ** 31 - 1
    out = (y < 0) | (y >= 333)
    A[out] = float("nan")
    A[0, 0] = float("inf")
    A[2, 50] = float("-inf")
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    _, row = pkg.softmax_head_loss(A, W, b, y)
    _check_all(A, W, b, y, loss, row, (dA, dW, db))
    assert float(loss[1]) == 0.0 and not dW[1].any() and not db[1].any()


@pytest.mark.parametrize("bf16", [False, True])
def test_no_rows(pkg, bf16):
    import torch
    A, W, b, y = _inputs(2, 1, 24, 40, bf16, 6)
    loss, dA, dW, db = pkg.softmax_head_grad(A[:, :0], W, b, y[:, :0], dW=torch.full_like(W, 3.0))
    l2, row = pkg.softmax_head_loss(A[:, :0], W, b, y[:, :0])
    torch.cuda.synchronize()
    assert not loss.any() and not l2.any() and dA.numel() == 0 and row.numel() == 0 and not dW.any() and not db.any()


@pytest.mark.parametrize("bf16", [False, True])
def test_classes_taken_out_by_the_bias(pkg, bf16):
    """-infinity: no share of the row, gradients finite; as a label: loss +infinity.  A whole part of 256 classes too.
    The type's lowest value does the same without infinities."""
    import torch
    A, W, b, y = _inputs(1, 20, 40, 700, bf16, 8)
    b[0, 256:512] = float("-inf")
    b[0, 5] = torch.finfo(torch.float32).min
    y[0] = torch.where((y[0] >= 256) & (y[0] < 512) | (y[0] == 5), 3, y[0])
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    _check_all_without(A, W, b, y, loss, dA, dW, db)
    assert not dW[0, :, 256:512].any() and not db[0, 256:512].any()
    y[0, 4] = 300
    loss, row = pkg.softmax_head_loss(A, W, b, y)
    _, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    assert float(loss[0]) == float("inf") and float(row[0, 4]) == float("inf") and bool(row[0, 5:].isfinite().all())
    assert bool(dA.isfinite().all()) and bool(dW.isfinite().all()) and bool(db.isfinite().all())


def _check_all_without(A, W, b, y, loss, dA, dW, db):
    """Against the same problem without the classes that are out."""
    import torch
    ok = b[0] > -1e30
    at = torch.cumsum(ok.long(), 0) - 1
    y2 = torch.where(y >= 0, at[y.clamp(min=0).long()].int(), y)
    _check_all(A, W[:, :, ok], b[:, ok], y2, loss, None, (dA, dW[:, :, ok], db[:, ok]))


@pytest.mark.parametrize("bf16", [False, True])
def test_well_fitted_rows(pkg, bf16):
    """p_y within 1e-6 of one: the label's delta keeps its digits."""
    import torch
    A, W, b, y = _inputs(1, 40, 64, 300, bf16, 9, scale=0.5)
    b[0, 7] += 14.0
    y[:] = 7
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    assert 0 < float(loss[0]) < 1e-2
    _check_all(A, W, b, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("bf16", [False, True])
def test_large_logits(pkg, bf16):
    A, W, b, y = _inputs(1, 30, 64, 600, bf16, 10, scale=60.0)
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    _check_all(A, W, b, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("off", [0, 1, 8])
def test_strides(pkg, bf16, off):
    """W inside rows of X, dW and db inside rows of G, activations with rows at a distance, one batch for all replicas."""
    import torch
    m, rows, d, classes = 3, 50, 72, 264
    A, W, b, y = _inputs(m, rows, d, classes, bf16, 12, 0.1)
    A = A[:1].expand(m, rows, d)
    big = torch.zeros(1, rows, 2 * d + off, device="cuda", dtype=A.dtype)
    big[:, :, off:off + d] = A[:1]
    Av = big[:, :, off:off + d].expand(m, rows, d)
    P = torch.full((m, off + d * classes + 64), 4.0, device="cuda", dtype=W.dtype)
    Wv = P[:, off:off + d * classes].view(m, d, classes) if off == 0 else P.as_strided((m, d, classes), (P.stride(0), classes, 1), off)
    Wv.copy_(W)
    G = torch.full((m, off + (d + 1) * classes + 64), 9.0, device="cuda")
    dWv = G.as_strided((m, d, classes), (G.stride(0), classes, 1), off)
    dbv = G.as_strided((m, classes), (G.stride(0), 1), off + d * classes)
    dAb = torch.full((m, rows, d + 8), 2.0, device="cuda", dtype=A.dtype)
    loss, dA, dW, db = pkg.softmax_head_grad(Av, Wv, b, y, dA=dAb[:, :, 3:3 + d], dW=dWv, db=dbv)
    _check_all(A, W, b, y, loss, None, (dA, dWv, dbv))
    assert bool((G[:, :off] == 9.0).all()) and bool((G[:, off + (d + 1) * classes:] == 9.0).all())
    assert bool((dAb[:, :, :3] == 2.0).all()) and bool((dAb[:, :, 3 + d:] == 2.0).all()) and bool((P[:, off + d * classes:] == 4.0).all())


def test_shared_weights(pkg):
    """One W for all replicas (distance 0), gradients of each."""
    A, W, b, y = _inputs(3, 40, 64, 520, True, 13)
    Ws, bs = W[:1].expand(3, 64, 520), b[:1].expand(3, 520)
    loss, dA, dW, db = pkg.softmax_head_grad(A, Ws, bs, y)
    _check_all(A, Ws, bs, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_in_chunks_and_replicas_in_groups(pkg, bf16):
    """More rows than are kept at a time (2 GB of exponentials), in all three ways: two chunks of rows, groups of replicas,
    and a replica whose rows of a chunk are all left out."""
    import torch
    classes, d = (200000, 8) if bf16 else (40000, 8)
    rows = 5600                      # 2.2 GB of fp16 exponentials; 2.2 GB of fp32 ones and deltas
    A, W, b, y = _inputs(1, rows, d, classes, bf16, 15, 0.05)
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    # 64-bit formulas over parts of the rows, with the mean over all
    kept = int((y >= 0).sum())
    part = [slice(k, min(rows, k + 700)) for k in range(0, rows, 700)]
    want, tol, wb, tb, ls, lt = 0, 0, 0, 0, 0, 0
    for s in part:
        r = _reference(A[0, s], W[0], b[0], y[0, s])
        n = max(1, int(r["keep"].sum()))
        _check("dA", dA[0, s][r["keep"]], r["dA"] * n / kept, r["dA_tol"] * n / kept, _half(dA))
        want, tol = want + r["dW"] * (n / kept), tol + r["dW_tol"] * (n / kept)
        wb, tb = wb + r["db"] * (n / kept), tb + r["db_tol"] * (n / kept)
        ls, lt = ls + r["loss"] * (n / kept), lt + r["loss_tol"] * (n / kept)
        del r
    _check("dW", dW[0], want, tol + rows * U * want.abs(), _half(dW))
    _check("db", db[0], wb, tb + rows * U * wb.abs(), _half(db))
    _check("loss", loss[0], ls, lt + 4 * U)
    del A, W, b, y, dA, dW, db, want, tol
    torch.cuda.empty_cache()
    m, classes = (40, 150000) if bf16 else (40, 30000)   # 256 rows of all replicas would be above 2 GB
    A, W, b, y = _inputs(m, 200, 8, classes, bf16, 16, 0.1)
    y[m - 1] = -1
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    for i in (0, 17, m - 2, m - 1):
        _check_all(A[i:i + 1], W[i:i + 1], b[i:i + 1], y[i:i + 1], loss[i:i + 1], None, (dA[i:i + 1], dW[i:i + 1], db[i:i + 1]))


def test_gradient_against_differences(pkg):
    import torch
    A, W, b, y = _inputs(2, 12, 20, 90, False, 17, 0.2)
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    keep = y >= 0

    def f(a, w, c):
        z = torch.stack([a[i] @ w[i] + c[i] for i in range(2)])
        row = torch.logsumexp(z, -1) - z.gather(-1, y.clamp(min=0).long()[..., None])[..., 0]
        return float(((row * keep).sum(1) / keep.sum(1)).sum())
    g = torch.Generator(device="cuda").manual_seed(2)
    base = [A.double(), W.double(), b.double()]
    for k, grad in enumerate((dA, dW, db)):
        v = torch.randn(base[k].shape, device="cuda", dtype=torch.float64, generator=g)
        h = 1e-5
        args = lambda s: [t + s * h * v if j == k else t for j, t in enumerate(base)]  # noqa: E731
        diff = (f(*args(1)) - f(*args(-1))) / (2 * h)
        assert abs(diff - float((grad.double() * v).sum())) <= 1e-5 * float((grad.double() * v).abs().sum()) + 1e-7


def test_streams_graph_and_repeats(pkg):
    import torch
    A, W, b, y = _inputs(2, 150, 136, 1234, True, 18, 0.1)
    ref = [t.clone() for t in pkg.softmax_head_grad(A, W, b, y)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pkg.softmax_head_grad(A, W, b, y, stream=side)
    here = pkg.softmax_head_grad(A, W, b, y)           # two calls at once, a workspace each
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, ref)) and all(torch.equal(p, q) for p, q in zip(here, ref))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pkg.softmax_head_grad(A, W, b, y)
        rows = pkg.softmax_head_loss(A, W, b, y)
    for k in range(3):
        A.copy_(A.flip(1))
        y[:, k::5] = -1 if k < 2 else 11               # the number of rows that count changes between replays
        graph.replay()
        torch.cuda.synchronize()
        want = pkg.softmax_head_grad(A, W, b, y)
        wrow = pkg.softmax_head_loss(A, W, b, y)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want)) and all(torch.equal(p, q) for p, q in zip(rows, wrow))


def test_bindings_refuse(pkg):
    import torch
    A, W, b, y = _inputs(2, 6, 16, 40, False, 19)
    bad = [lambda: pkg.softmax_head_grad(A, W.bfloat16(), b, y), lambda: pkg.softmax_head_grad(A, W, b, y.long()),
           lambda: pkg.softmax_head_grad(A, W, b[:, :39], y), lambda: pkg.softmax_head_grad(A, W[:1], b, y),
           lambda: pkg.softmax_head_grad(A, W.transpose(1, 2).contiguous().transpose(1, 2), b, y),
           lambda: pkg.softmax_head_grad(A, W, b, y, dW=W[:1].expand(2, 16, 40)), lambda: pkg.softmax_head_loss(A.half(), W.half(), b, y),
           lambda: pkg.softmax_head_grad(A, W, b, y, grad_dtype=torch.float16), lambda: pkg.softmax_head_loss(A, W, b, y[:, ::2])]
    for f in bad:
        with pytest.raises(pkg.LcError):
            f()


def test_more_replicas_than_a_launch_has_threads_for(pkg):
    import torch
    m, d, classes = 65535, 1030, 3
    A, W, b, y = _inputs(m, 1, d, classes, False, 41)
    loss, dA, dW, db = pkg.softmax_head_grad(A, W, b, y)
    for i in (0, 1, 4095, 8011, 8012, 40000, m - 1):
        want = _reference(A[i], W[i], b[i], y[i])
        _check("loss", loss[i], want["loss"], want["loss_tol"])
        _check("dA", dA[i], want["dA"], want["dA_tol"])
        _check("dW", dW[i], want["dW"], want["dW_tol"])
        _check("db", db[i], want["db"], want["db_tol"])
    ref = torch.nn.functional.cross_entropy((A[:, 0, :, None] * W).sum(1) + b, y[:, 0].long(), reduction="none")
    assert torch.allclose(loss, ref, rtol=1e-3, atol=1e-3)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows", [1, 70, 300, 520])
def test_what_stands_between_rows_of_the_weights_is_not_used(pkg, bf16, rows):
    """Every length of a row's end, rows of W at odd distances with NaN between and around them."""
    import torch
    m, d = 2, 45
    for k, classes in enumerate((8, 9, 15, 23, 31, 33, 63, 66, 127, 129, 130, 255, 259, 268)):
        A, W, b, y = _inputs(m, rows, d, classes, bf16, 50 + k, 0.1)
        off, row = 1 + k % 8, classes + 1 + k % 5
        P = torch.full((m, off + d * row + 16), float("nan"), device="cuda", dtype=W.dtype)
        Wv = P.as_strided((m, d, classes), (P.stride(0), row, 1), off)
        Wv.copy_(W)
        loss, row_loss = pkg.softmax_head_loss(A, Wv, b, y)
        _check_all(A, W, b, y, loss, row_loss)
        loss, dA, dW, db = pkg.softmax_head_grad(A, Wv, b, y)
        _check_all(A, W, b, y, loss, None, (dA, dW, db))


def test_shared_fp32_weights(pkg):
    A, W, b, y = _inputs(3, 40, 64, 520, False, 14)
    Ws, bs = W[:1].expand(3, 64, 520), b[:1].expand(3, 520)
    loss, dA, dW, db = pkg.softmax_head_grad(A, Ws, bs, y)
    _check_all(A, Ws, bs, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("rows", [1, 66, 300])
def test_fp32_weights_split_on_their_way(pkg, rows):
    """As many weights as that is done for, at every alignment of 4 bytes."""
    import torch
    m, d = 5, 130
    for k, classes in enumerate((10000, 10001, 10003, 10126)):
        A, W, b, y = _inputs(m, rows, d, classes, False, 70 + k, 0.1)
        row = classes + k
        P = torch.full((m, 16 + d * row), float("nan"), device="cuda")
        Wv = P.as_strided((m, d, classes), (P.stride(0), row, 1), 1 + k)
        Wv.copy_(W)
        loss, row_loss = pkg.softmax_head_loss(A, Wv, b, y)
        _check_all(A, W, b, y, loss, row_loss)
        loss, dA, dW, db = pkg.softmax_head_grad(A, Wv, b, y)
        _check_all(A, W, b, y, loss, None, (dA, dW, db))


@pytest.mark.parametrize("classes", [1000, 40003])
def test_captured_fp32_gradients(pkg, classes):
    """Weights copied in parts and split in place; replays with other inputs."""
    import torch
    A, W, b, y = _inputs(3, 40, 72, classes, False, 90, 0.1)
    pkg.softmax_head_grad(A, W, b, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pkg.softmax_head_grad(A, W, b, y)
    for k in range(3):
        A2, W2, b2, y2 = _inputs(3, 40, 72, classes, False, 91 + k, 0.3)
        for to, new in ((A, A2), (W, W2), (b, b2), (y, y2)):
            to.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = pkg.softmax_head_grad(A, W, b, y)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
        _check_all(A, W, b, y, got[0], None, got[1:])
