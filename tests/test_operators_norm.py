"""Layer norm and its gradients against the formulas in 64 bits (GPU).

Tolerances.  u = 2^-24, n the elements of a row, L = n / 8 + 16 additions that a value passes on its way into a sum of a row at most.  With X = max |x - mean| of the
row and s its standard deviation (sqrt(var + eps)), every centred value is off by at most u (2 |mean u n| + 4 X) + the error of the mean in two
parts, (L + 4) u mean|c| <= (L + 4) u X, so h = c / s by dc / s + |h| (L + 8) u; eight roundings of 32 bits more for products and sums, and half a step of
the result's type.  dx = r (g - A - h B) with A, B means over the row: their sums are off by (L + 8) u of the mean magnitudes.
dw, db: up to 128 + 40 additions in 32 bits, u each of the sum of magnitudes, beside what h is off by."""
import math

import pytest

pytestmark = pytest.mark.gpu

# (rows, n): one of everything, less than a vector, every team of lanes with and without a tail, rows of a block, more rows than blocks, long rows
SIZES = [(1, 1), (5, 1), (3, 2), (33, 7), (257, 8), (100, 61), (70, 64), (9, 65), (131, 128), (17, 130), (65, 257), (40, 512), (33, 515), (21, 1021), (12, 1024), (9, 1030),
         (14, 2048), (7, 2051), (13, 4096), (6, 4104), (5, 8192), (4, 8200), (3, 16384), (4, 16390), (2, 32768), (2, 32771), (3, 70001), (20000, 24), (3001, 200), (1500, 1100)]
KINDS = [("float32", "float32"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float16"), ("float16", "float32")]


def half(t):
    import torch
    return torch.finfo(t).eps / 2


def padded(t, before, after):
    """t as a part of a larger tensor whose other elements are NaN."""
    import torch
    big = torch.full((t.shape[0] + 2, t.shape[1] + before + after), math.nan, dtype=t.dtype, device=t.device)
    big[1:-1, before:before + t.shape[1]] = t
    return big[1:-1, before:before + t.shape[1]]


def make(rows, n, kind, params, seed, mean=0.5, spread=1.0):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda:0")  # noqa: E731
    T, W = getattr(torch, kind), getattr(torch, params)
    return (spread * rand(rows, n) + mean).to(T), (1 + 0.3 * rand(n)).to(W), (0.2 * rand(n)).to(W), rand(rows, n).to(T)


def reference(x, w, b, dy, eps):
    """Values and their bounds: y, dx, dw, db."""
    import torch
    rows, n = x.shape
    u, L = 2.0 ** -24, n / 8 + 16
    hx = half(x.dtype)
    hw = hx if w is None else half(w.dtype)
    tiny = {torch.float16: 2.0 ** -25, torch.bfloat16: 1e-38, torch.float32: 1e-38}          # half a step of the subnormal numbers
    tx, tw = tiny[x.dtype], tiny[x.dtype if w is None else w.dtype]
    x, dy = x.double(), dy.double()
    w = torch.ones(n, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(n, dtype=torch.float64, device=x.device) if b is None else b.double()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    s = torch.sqrt((c * c).mean(1, keepdim=True) + eps)
    h = c / s
    X = c.abs().amax(1, keepdim=True)
    # c = x - m1 is one rounding of c + (m1's own error, <= (L + 2) u mean|x|), which m2 takes off again
    first = (L + 2) * u * x.abs().mean(1, keepdim=True)
    dc = u * (c.abs() + first) + (L + 4) * u * (X + first) + 2 * u * first + 2 * u * c.abs()
    dh = dc / s + h.abs() * (L + 10) * u
    y = h * w + b
    out = {"y": (y, 1.01 * (hx * y.abs() + dh * w.abs() + 3 * u * ((h * w).abs() + b.abs())) + tx)}
    g = dy * w
    A, B = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    dA = (L + 8) * u * g.abs().mean(1, keepdim=True)
    dB = (L + 8) * u * (g * h).abs().mean(1, keepdim=True) + (g.abs() * dh).mean(1, keepdim=True)
    dx = (g - A - h * B) / s
    size = (g.abs() + A.abs() + (h * B).abs()) / s
    out["dx"] = (dx, 1.02 * (hx * dx.abs() + (dA + dB * h.abs() + dh * B.abs()) / s + (L + 16) * u * size) + tx)
    dw, db = (dy * h).sum(0), dy.sum(0)
    out["dw"] = (dw, 1.01 * (hw * dw.abs() + (dy.abs() * dh).sum(0) + 170 * u * (dy * h).abs().sum(0)) + tw)
    out["db"] = (db, 1.01 * (hw * db.abs() + 170 * u * dy.abs().sum(0)) + tw)
    return out


def close(name, got, want):
    import torch
    value, bound = want
    off = (got.double() - value).abs()
    assert got.shape == value.shape and torch.isfinite(got).all(), name
    worst = float((off / bound).max()) if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3f of the bound" % (name, worst)


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind,params", KINDS)
def test_forward_and_gradients(size, kind, params):
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(*size, kind, params, size[0] * 7919 + size[1])
    for weight, bias in ((w, b), (w, None), (None, None)):
        want = reference(x, weight, bias, dy, 1e-5)
        y, stats = P.layer_norm_forward(x, weight, bias)
        close("y", y, want["y"])
        assert torch.equal(P.layer_norm(x, weight, bias), y)
        dx, dw, db = P.layer_norm_gradients(dy, x, weight, stats)
        close("dx", dx, want["dx"])
        assert dx.dtype == x.dtype
        if weight is None:
            assert dw is None and db is None
        else:
            assert dw.dtype == db.dtype == weight.dtype
            close("dw", dw, want["dw"])
            close("db", db, want["db"])


@pytest.mark.parametrize("kind,params", KINDS)
def test_autograd_and_needs(kind, params):
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(37, 100, kind, params, 1)
    y, stats = P.layer_norm_forward(x, w, b, eps=1e-3)
    all3 = P.layer_norm_gradients(dy, x, w, stats)
    for needed in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (False, False, False)):
        for got, full, asked in zip(P.layer_norm_gradients(dy, x, w, stats, need=needed), all3, needed):
            assert torch.equal(got, full) if asked else got is None
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    for _ in range(2):
        z = P.layer_norm(*leaves, eps=1e-3)
        assert torch.equal(z, y)
        for got, full in zip(torch.autograd.grad(z, leaves, dy), all3):
            assert torch.equal(got, full)
    only = x.clone().requires_grad_()
    assert torch.equal(torch.autograd.grad(P.layer_norm(only, w, b, eps=1e-3), only, dy)[0], all3[0])
    assert P.layer_norm(only, eps=1e-3).requires_grad
    # more than two dimensions
    assert torch.equal(P.layer_norm(x[:36].reshape(3, 4, 3, 100), w, b, eps=1e-3).reshape(36, 100), y[:36])
    assert torch.equal(P.layer_norm(x[5], w, b, eps=1e-3), y[5])


@pytest.mark.parametrize("kind,params", KINDS)
@pytest.mark.parametrize("size", [(9, 13), (21, 64), (6, 1023), (4, 4100), (2, 33000)], ids=str)
def test_strides_and_neighbours(kind, params, size):
    """Rows inside of larger tensors, dy of another stride, dy and x that autograd expands or transposes; what lies around is not touched."""
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(*size, kind, params, 2)
    y, stats = P.layer_norm_forward(x, w, b)
    grads = P.layer_norm_gradients(dy, x, w, stats)
    for before, after in ((1, 0), (3, 5), (8, 8)):
        xp, dp = padded(x, before, after), padded(dy, after, before)
        wp, bp = (padded(t[None], before, after)[0] for t in (w, b))
        yp, sp = P.layer_norm_forward(xp, wp, bp)
        assert torch.equal(yp, y) and torch.equal(sp, stats)
        for got, want in zip(P.layer_norm_gradients(dp, xp, wp, sp), grads):
            assert torch.equal(got, want)
    xt = x.t().contiguous().t()                              # copied
    assert torch.equal(P.layer_norm(xt, w, b), y)
    one = dy[:1].expand_as(dy)                               # the gradient of a sum over rows: a stride of 0
    for got, want in zip(P.layer_norm_gradients(one, x, w, stats), P.layer_norm_gradients(one.contiguous(), x, w, stats)):
        assert torch.equal(got, want)
    every = x.repeat_interleave(2, 1)[:, ::2]                # an inner stride of 2
    assert torch.equal(P.layer_norm(every, w, b), y)


@pytest.mark.parametrize("n", [1, 5, 64, 1000, 3001, 9000, 40000])
def test_a_mean_far_away(n):
    """fp32 rows whose mean is 10^4 standard deviations from 0: 10^-3 of y where the mean is one number of 32 bits."""
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(5, n, "float32", "float32", 3, mean=1e4)
    want = reference(x, w, b, dy, 1e-5)
    y, stats = P.layer_norm_forward(x, w, b)
    close("y", y, want["y"])
    grads = P.layer_norm_gradients(dy, x, w, stats)
    for name, got in zip(("dx", "dw", "db"), grads):
        close(name, got, want[name])
    if n >= 64:
        off = (y.double() - want["y"][0]).abs().max() / want["y"][0].abs().max()
        assert float(off) < 2e-5                             # 4 u 1e4 of the first mean's own error would be 2e-3


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [16, 1000, 5000, 40000])
def test_large_and_small_values(kind, n):
    """Squares that 32 bits do not hold, and rows of nearly one value."""
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(6, n, kind, "float32", 4, mean=0.0)
    scale = torch.tensor([1e25, 1e30, 1e37, 1e-3, 1e-15, 1.0], device="cuda:0")[:, None]
    xs = (x.float() * scale).to(x.dtype)
    y, stats = P.layer_norm_forward(xs, w, b)
    want = reference(xs, w, b, dy, 1e-5)
    close("y", y, want["y"])
    dx, dw, db = P.layer_norm_gradients(dy, xs, w, stats)
    value, bound = want["dx"]
    assert ((dx.double() - value).abs() <= bound + 2e-38).all()      # results under 2^-126 for the first rows
    close("dw", dw, want["dw"])
    same = torch.full((3, n), 7.0, dtype=x.dtype, device="cuda:0")
    y, stats = P.layer_norm_forward(same, w, b)
    assert torch.equal(y, b.to(x.dtype).expand_as(y))
    dx, dw, _ = P.layer_norm_gradients(dy[:3], same, w, stats)
    assert torch.isfinite(dx).all() and not dw.any()


@pytest.mark.parametrize("n", [7, 100, 1024, 9000, 40000])
def test_values_that_are_not_finite_stay_in_their_row(n):
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(40, n, "bfloat16", "bfloat16", 5)
    y, stats = P.layer_norm_forward(x, w, b)
    dx, dw, db = P.layer_norm_gradients(dy, x, w, stats)
    bad = x.clone()
    bad[3, n // 2], bad[17, 0], bad[39, n - 1] = math.nan, math.inf, -math.inf
    yb, sb = P.layer_norm_forward(bad, w, b)
    dxb, dwb, dbb = P.layer_norm_gradients(dy, bad, w, sb)
    rows = torch.ones(40, dtype=torch.bool)
    rows[[3, 17, 39]] = False
    assert torch.equal(yb[rows], y[rows]) and torch.equal(dxb[rows], dx[rows]) and torch.equal(dbb, db)
    assert yb[~rows].isnan().all() and dxb[~rows].isnan().all() and dwb.isnan().all()


def test_no_rows():
    import torch
    import paper_1710_06952_amd as P
    x, w = torch.zeros(0, 100, device="cuda:0"), torch.ones(100, device="cuda:0")
    y, stats = P.layer_norm_forward(x, w, w)
    dx, dw, db = P.layer_norm_gradients(x, x, w, stats)
    assert y.shape == dx.shape == (0, 100) and not dw.any() and not db.any() and dw.shape == (100,)


def test_against_differences():
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(3, 50, "float32", "float32", 6)
    _, stats = P.layer_norm_forward(x, w, b)
    grads = P.layer_norm_gradients(dy, x, w, stats)
    loss = lambda *p: (torch.nn.functional.layer_norm(p[0], (50,), p[1], p[2], 1e-5) * dy.double()).sum()  # noqa: E731
    args = [t.double() for t in (x, w, b)]
    for i, g in enumerate(grads):
        for at in (0, 17, 49):
            plus, minus = [t.clone() for t in args], [t.clone() for t in args]
            plus[i].view(-1)[at] += 1e-4
            minus[i].view(-1)[at] -= 1e-4
            slope = float((loss(*plus) - loss(*minus)) / 2e-4)
            assert abs(slope - float(g.view(-1)[at])) < 1e-6 + 1e-5 * abs(slope)     # 1e-8 of the third derivative, and 50 roundings of 32 bits


def test_another_stream_and_a_graph():
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dy = make(300, 520, "bfloat16", "float32", 7)
    y, stats = P.layer_norm_forward(x, w, b)
    grads = P.layer_norm_gradients(dy, x, w, stats)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2, stats2 = P.layer_norm_forward(x, w, b)
        grads2 = P.layer_norm_gradients(dy, x, w, stats2)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(grads, grads2))
    xs, ds = x.clone(), dy.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        yg, sg = P.layer_norm_forward(xs, w, b)
        gg = P.layer_norm_gradients(ds, xs, w, sg)
    with torch.cuda.graph(torch.cuda.CUDAGraph()), pytest.raises(RuntimeError, match="captured"):
        P.layer_norm(xs.requires_grad_(), w, b)
    xs.requires_grad_(False)
    for turn in range(4):
        new, dnew = make(300, 520, "bfloat16", "float32", 20 + turn)[::3]
        xs.copy_(new)
        ds.copy_(dnew)
        graph.replay()
        torch.cuda.synchronize()
        y, stats = P.layer_norm_forward(new, w, b)
        assert torch.equal(yg, y)
        for got, want in zip(gg, P.layer_norm_gradients(dnew, new, w, stats)):
            assert torch.equal(got, want)
