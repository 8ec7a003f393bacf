"""lc_layer_norm and lc_layer_norm_grad against the formulas in 64 bits.

Tolerances.  u = 2^-24.  A sum of n values in 32 bits, formed in parts of a thread, a wavefront and a workgroup, is off
by at most d u sum |.| with d its depth; d <= 32 (a thread's values) + 6 + 4, and for rows beyond the registers n / 256
more.  The mean is then off by d u mean|x|, n = (x - mean) r by that times r plus 4 u |n| and, through the variance,
d u |n|.  Results in bf16 add half a step, 2^-8 |.|; fp32 rounds as part of the 4 u."""
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


def _inputs(m, rows, cols, dtype, seed, offset=0.3):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x = (rn(m, rows, cols) * 1.5 + offset).to(dtype)
    return x, rn(m, rows, cols).to(dtype), 1 + 0.1 * rn(m, cols), 0.1 * rn(m, cols)


def _reference(x, dy, gain, bias, eps):
    import torch
    x, dy = x.double(), dy.double()
    g = gain.double()[:, None] if gain is not None else torch.ones_like(x[:, :1])
    b = bias.double()[:, None] if bias is not None else torch.zeros_like(x[:, :1])
    mean = x.mean(-1, keepdim=True)
    r = ((x - mean).pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    n = (x - mean) * r
    h = dy * g
    dx = r * (h - h.mean(-1, keepdim=True) - n * (h * n).mean(-1, keepdim=True))
    return dict(y=n * g + b, mean=mean, r=r, n=n, h=h, dx=dx, dgain=(dy * n).sum(1), dbias=dy.sum(1), dy=dy, g=g, b=b, x=x)


def _check(name, got, want, tol):
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), (name, float((off - tol).max()), float(off.max()))


def _check_all(pkg, x, dy, gain, bias, eps, grad=True):
    import torch
    m, rows, cols = x.shape
    print(f"layer norm m={m} rows={rows} cols={cols} {x.dtype} strides={x.stride()}", flush=True)
    w = _reference(x, dy, gain, bias, eps)
    half = torch.finfo(torch.bfloat16).eps / 2 if x.dtype == torch.bfloat16 else 0.0
    d = 42 + (cols / 256 if cols > 8192 else 0)
    y, stats = pkg.layer_norm(x, gain, bias, eps)
    torch.cuda.synchronize()
    size = w["x"].abs().mean(-1, keepdim=True)
    e_mean = d * U * size
    e_n = e_mean * w["r"] + (4 + d) * U * w["n"].abs()
    _check("mean", stats[..., :1], w["mean"], e_mean + U * w["mean"].abs())
    # the variance: its own sum, and twice the mean's error against the largest difference
    _check("r", stats[..., 1:], w["r"], w["r"] * (d + 4) * U + w["r"] ** 2 * e_mean * 2)
    e_y = e_n * w["g"].abs() + 2 * U * (w["n"] * w["g"]).abs() + U * w["b"].abs()
    _check("y", y, w["y"], e_y + half * (w["y"].abs() + e_y) + 1e-37)
    if not grad:
        return
    # the backward pass from the 64-bit statistics as fp32, so that only its own error counts
    st = torch.cat([w["mean"], w["r"]], -1).float()
    dx, dg, db = pkg.layer_norm_grad(x, dy, gain, st)
    torch.cuda.synchronize()
    e_n = w["r"] * U * (w["x"].abs() + w["mean"].abs()) + 4 * U * w["n"].abs()
    ah, an = w["h"].abs(), w["n"].abs()
    e_c1 = (d + 2) * U * ah.mean(-1, keepdim=True)
    e_c2 = (d + 4) * U * (ah * an).mean(-1, keepdim=True) + (ah * e_n).mean(-1, keepdim=True)
    c2 = (w["h"] * w["n"]).mean(-1, keepdim=True).abs()
    e_dx = w["r"] * (e_c1 + an * e_c2 + e_n * c2 + 6 * U * (ah + ah.mean(-1, keepdim=True) + an * c2))
    _check("dx", dx, w["dx"], e_dx + half * (w["dx"].abs() + e_dx) + 1e-37)
    # over the rows: at most all of them in one thread, then the workgroups' partial sums
    deep = min(rows, 16384) + 12
    _check("dgain", dg, w["dgain"], deep * U * (w["dy"].abs() * an).sum(1) + (w["dy"].abs() * e_n).sum(1) + 1e-37)
    _check("dbias", db, w["dbias"], deep * U * w["dy"].abs().sum(1) + 1e-37)


SIZES = [(1, 1, 1), (2, 3, 5), (3, 17, 64), (4, 32, 256), (2, 5, 511), (1, 9, 512), (2, 33, 513), (5, 100, 1500), (2, 7, 2048),
         (1, 3, 2049), (2, 5, 4096), (1, 6, 4104), (1, 5, 8192), (2, 3, 8193), (1, 2, 20000), (64, 4, 8), (1, 5000, 48), (3, 1100, 130)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("m,rows,cols", SIZES)
def test_sizes(pkg, m, rows, cols, bf16):
    import torch
    x, dy, gain, bias = _inputs(m, rows, cols, torch.bfloat16 if bf16 else torch.float32, m + rows + cols)
    _check_all(pkg, x, dy, gain, bias, 1e-5)


@pytest.mark.parametrize("bf16", [False, True])
def test_values(pkg, bf16):
    """A large offset (no cancellation in the variance), constant rows (variance 0: r = 1 / sqrt(eps)), no gain or bias."""
    import torch
    t = torch.bfloat16 if bf16 else torch.float32
    x, dy, gain, bias = _inputs(2, 12, 300, t, 3, offset=1000.0)
    _check_all(pkg, x, dy, gain, bias, 1e-5)
    _check_all(pkg, x, dy, None, bias, 1e-5)
    _check_all(pkg, x, dy, gain, None, 1e-5, grad=False)
    _check_all(pkg, x, dy, None, None, 0.0, grad=False)
    x = torch.full((1, 4, 256), 3.0, device="cuda", dtype=t)   # an exact mean
    y, st = pkg.layer_norm(x, None, None, 1e-4)
    assert float(y.abs().max()) == 0.0 and bool((st[..., 0] == 3.0).all())
    assert bool(((st[..., 1] - 100.0).abs() < 100 * 2.0 ** -20).all())


def test_not_finite_stays_in_its_row(pkg):
    import torch
    x, dy, gain, bias = _inputs(2, 8, 700, torch.float32, 5)
    y0, _ = pkg.layer_norm(x, gain, bias)
    x[0, 3, 10] = float("nan")
    x[1, 5, 0] = float("inf")
    y, _ = pkg.layer_norm(x, gain, bias)
    bad = torch.zeros(2, 8, dtype=torch.bool, device="cuda")
    bad[0, 3] = bad[1, 5] = True
    assert bool(y[bad].isnan().all()) and bool((y[~bad] == y0[~bad]).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cols", [256, 300, 8200])
def test_strides_and_places(pkg, cols, bf16):
    """Rows at a distance, replicas interleaved, unaligned starts, parameters inside rows of a larger array, results
    where the input stands; what lies between rows keeps its values."""
    import torch
    t = torch.bfloat16 if bf16 else torch.float32
    m, rows = 3, 10
    x, dy, gain, bias = _inputs(m, rows, cols, t, 11)
    want, st = pkg.layer_norm(x, gain, bias)
    wdx, wdg, wdb = pkg.layer_norm_grad(x, dy, gain, st)
    for off in (0, 1, 8):
        big = torch.full((rows, m, cols + 24), 7.0, device="cuda", dtype=t)
        v = big.transpose(0, 1)[:, :, off:off + cols]      # replicas inside a row
        v.copy_(x)
        P = torch.full((m, 2 * cols + 64), 5.0, device="cuda")
        P[:, 3:3 + cols] = gain
        P[:, 3 + cols:3 + 2 * cols] = bias
        G = torch.full_like(P, 9.0)
        gain_v, bias_v = P[:, 3:3 + cols], P[:, 3 + cols:3 + 2 * cols]
        out, st2 = pkg.layer_norm(v, gain_v, bias_v)
        # the same values: vector and element access add in another order, at most a step apart
        near = lambda a, b: bool(((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-5).all()) if bf16 else \
            bool(((a - b).abs() <= 1e-5 * (1 + b.abs())).all())  # noqa: E731
        assert near(out, want) and near(st2, st)
        pkg.layer_norm(v, gain_v, bias_v, out=v)           # in place
        assert bool((v == out).all())
        rest = big.clone()
        rest[:, :, off:off + cols] = 7.0
        assert bool((rest == 7.0).all())
        v.copy_(x)
        dxv = torch.full_like(big, 7.0).transpose(0, 1)[:, :, off:off + cols]
        dxv.copy_(dy)
        _, dg, db = pkg.layer_norm_grad(v, dxv, gain_v, st, dx=dxv, dgain=G[:, 3:3 + cols], dbias=G[:, 3 + cols:3 + 2 * cols])
        assert near(dxv, wdx) and near(dg, wdg) and near(db, wdb)
        assert bool((G[:, :3] == 9.0).all()) and bool((G[:, 3 + 2 * cols:] == 9.0).all())


def test_gradient_against_differences(pkg):
    """dx, dgain and dbias as directional derivatives of sum(y * w), central differences in 64 bits of the formula."""
    import torch
    x, w, gain, bias = _inputs(2, 6, 40, torch.float32, 21)
    _, st = pkg.layer_norm(x, gain, bias, 1e-5)
    dx, dg, db = pkg.layer_norm_grad(x, w, gain, st)

    def f(x, gain, bias):
        mean = x.mean(-1, keepdim=True)
        r = ((x - mean).pow(2).mean(-1, keepdim=True) + 1e-5).rsqrt()
        return float((((x - mean) * r * gain[:, None] + bias[:, None]) * w.double()).sum())
    g = torch.Generator(device="cuda").manual_seed(1)
    X, Ga, Bi = x.double(), gain.double(), bias.double()
    for k, (grad, base) in enumerate(((dx, X), (dg, Ga), (db, Bi))):
        v = torch.randn(base.shape, device="cuda", dtype=torch.float64, generator=g)
        h = 1e-5
        args = lambda s: [b + s * h * v if j == k else b for j, b in enumerate((X, Ga, Bi))]  # noqa: E731
        diff = (f(*args(1)) - f(*args(-1))) / (2 * h)
        # fp32 gradients: 1e-5 of the sum of magnitudes; differences: h^2 and 64-bit noise / h, both below 1e-8
        assert abs(diff - float((grad.double() * v).sum())) <= 1e-5 * float((grad.double() * v).abs().sum()) + 1e-6


def test_no_rows(pkg):
    import torch
    x = torch.empty(2, 0, 16, device="cuda")
    y, st = pkg.layer_norm(x)
    assert y.shape == x.shape and st.shape == (2, 0, 2)
    _, dg, db = pkg.layer_norm_grad(x, x, None, st, dgain=torch.ones(2, 16, device="cuda"), dbias=torch.ones(2, 16, device="cuda"))
    assert not dg.any() and not db.any()


def test_streams_graph_and_repeats(pkg):
    """On a stream that is not the current one, captured and replayed with other calls between the replays, always the same bits."""
    import torch
    x, dy, gain, bias = _inputs(4, 300, 700, torch.bfloat16, 31)
    y0, st0 = pkg.layer_norm(x, gain, bias)
    ref = [t.clone() for t in pkg.layer_norm_grad(x, dy, gain, st0)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, st = pkg.layer_norm(x, gain, bias, stream=side)
    got = pkg.layer_norm_grad(x, dy, gain, st, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y0) and all(torch.equal(a, b) for a, b in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gy, gst = pkg.layer_norm(x, gain, bias)
        gg = pkg.layer_norm_grad(x, dy, gain, gst)
    for k in range(3):
        x.mul_(1 + 0.25 * k)
        graph.replay()
        torch.cuda.synchronize()
        y, st = pkg.layer_norm(x, gain, bias)
        want = pkg.layer_norm_grad(x, dy, gain, st)
        torch.cuda.synchronize()
        assert torch.equal(gy, y) and torch.equal(gst, st) and all(torch.equal(a, b) for a, b in zip(gg, want))


def test_bindings_refuse(pkg):
    import torch
    x, dy, gain, bias = _inputs(2, 3, 8, torch.float32, 1)
    _, st = pkg.layer_norm(x, gain, bias)
    bad = [lambda: pkg.layer_norm(x.half()), lambda: pkg.layer_norm(x[0]), lambda: pkg.layer_norm(x, gain.double()),
           lambda: pkg.layer_norm(x, gain[:, :7]), lambda: pkg.layer_norm(x, gain.cpu()), lambda: pkg.layer_norm(x.transpose(1, 2)),
           lambda: pkg.layer_norm(x, out=torch.empty(2, 3, 9, device="cuda")), lambda: pkg.layer_norm(x, eps=-1.0),
           lambda: pkg.layer_norm(x, out=x[:1].expand(2, 3, 8)), lambda: pkg.layer_norm_grad(x, dy.bfloat16(), gain, st),
           lambda: pkg.layer_norm_grad(x, dy, gain, st[:1])]
    for f in bad:
        with pytest.raises(pkg.LcError):
            f()
