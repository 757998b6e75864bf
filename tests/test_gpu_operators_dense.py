"""Dense layers and their gradients against the formulas in 64 bits (GPU).

Tolerances, for products of `n` terms whose magnitudes sum to S: n + 8 roundings to 32 bits, (n + 8) 2^-24 S, and one rounding to the type,
half a step of it.  Activations and slopes are within 5e-6 (the tail of gelu is fitted to 2.6e-6, the reciprocal and exponential of
the instruction set add a few 2^-23); a slope is kept in steps of 2^-15; |act'| <= 1.13, |act''| <= 1.2."""
import math

import pytest

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "silu"]
# (M, K, N): one of everything, odd sizes, ends inside tiles and vectors, few rows, split sums, tiles of 64, 128 and 256
SIZES = [(1, 1, 1), (1, 8, 64), (3, 7, 5), (2, 64, 9), (16, 8, 520), (64, 784, 1024), (130, 257, 391), (257, 63, 129), (300, 1000, 10), (33, 2049, 65),
         (1, 4096, 768), (5, 4100, 72), (40, 6, 1000), (1100, 200, 2000), (1101, 203, 2001), (2049, 72, 4100), (2100, 1030, 4097), (2056, 72, 4104),
         (2952, 2824, 3096), (1701, 1703, 1705), (256, 8192, 256), (520, 4096, 392), (72, 1024, 8192), (8192, 136, 264), (47, 6060, 477), (3, 8191, 66), (64, 5000, 40)]


def half(t):
    import torch
    return torch.finfo(t).eps / 2


def padded(t, before, after):
    """t as a part of a larger tensor whose other elements are NaN."""
    import torch
    big = torch.full((t.shape[0] + 2, t.shape[1] + before + after), math.nan, dtype=t.dtype, device=t.device)
    big[1:-1, before:before + t.shape[1]] = t
    return big[1:-1, before:before + t.shape[1]]


def make(M, K, N, dtype, layout, seed, pad=(0, 0)):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda:0")  # noqa: E731
    place = lambda t: padded(t.to(dtype), *pad) if pad != (0, 0) else t.to(dtype)  # noqa: E731
    x, r, dy = place(rand(M, K)), place(rand(M, N)), place(rand(M, N))
    w = rand(N, K) / math.sqrt(K)
    w = place(w) if layout == "nk" else place(w.t().contiguous()).t()
    b = (0.5 * rand(N)).to(dtype)
    return x, w, b, r, dy


def activation(z, act):
    """act(z), act'(z) in 64 bits"""
    import torch
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return z * s, s * (1 + z * (1 - s))


def reference(x, w, b, r, dy, act):
    """Values and their bounds: y, dx, dw, db."""
    import torch
    M, K = x.shape
    N = w.shape[0]
    h, u = half(x.dtype), 2.0 ** -24
    x, w, dy = x.double(), w.double().contiguous(), dy.double()
    b = torch.zeros(N, dtype=torch.float64, device=x.device) if b is None else b.double()
    r = torch.zeros(M, N, dtype=torch.float64, device=x.device) if r is None else r.double()
    z = torch.mm(x, w.t().contiguous()) + b
    size = torch.mm(x.abs(), w.abs().t().contiguous()) + b.abs()
    zerr = (K + 8) * u * size
    a, s = activation(z, act)
    y = a + r
    aerr = 1.13 * zerr + (0 if act == "none" else 5e-6 * a.abs() + 1e-30)
    out = {"y": (y, 1.01 * h * y.abs() + 1.01 * (aerr + 2 * u * (a.abs() + r.abs())) + 1e-30)}
    serr = torch.zeros_like(z)
    if act == "relu":
        serr = (z.abs() <= zerr).double()
    elif act != "none":
        serr = 1.01 * 2.0 ** -16 + 5e-6 + 1.2 * zerr
    dz = dy * s
    dzerr = dy.abs() * serr + 2 * u * dz.abs()
    rounded = dzerr + (0 if act == "none" else 1.01 * h * (dz.abs() + dzerr) + 2.0 ** -25 * (x.dtype != torch.bfloat16))
    tiny = torch.finfo(torch.float16).smallest_normal * half(torch.float16) if h == half(torch.float16) else 0.0    # subnormal results
    mm = lambda p, q: torch.mm(p, q.contiguous())  # noqa: E731
    dx, dw, db = mm(dz, w), mm(dz.t().contiguous(), x), dz.sum(0)
    out["dx"] = (dx, 1.01 * h * dx.abs() + 1.01 * (mm(rounded, w.abs()) + (N + 8) * u * mm(dz.abs(), w.abs())) + tiny + 1e-30)
    out["dw"] = (dw, 1.01 * h * dw.abs() + 1.01 * (mm(rounded.t().contiguous(), x.abs()) + (M + 8) * u * mm(dz.abs().t().contiguous(), x.abs())) + tiny + 1e-30)
    out["db"] = (db, 1.01 * h * db.abs() + 1.01 * (dzerr.sum(0) + 16 * u * dz.abs().sum(0)) + tiny + 1e-30)
    return out


def close(name, got, want):
    import torch
    value, bound = want
    off = (got.double() - value).abs()
    assert got.shape == value.shape and torch.isfinite(got).all(), name
    worst = float((off / bound).max()) if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3f of the bound" % (name, worst)


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_forward_and_gradients(size, dtype, layout):
    import torch
    import paper_1710_06952_amd as P
    M, K, N = size
    for n, act in enumerate(ACTS):
        if n > 1 and M * N > 2_000_000:                  # the large ones once with an activation of each kind
            continue
        print(size, dtype, layout, act, flush=True)
        x, w, b, r, dy = make(M, K, N, getattr(torch, dtype), layout, seed=M + K + N + n)
        b, r = (b, r) if n % 2 == 0 else (None, None) if n == 1 else (b, None)
        want = reference(x, w, b, r, dy, act)
        close("y without gradients", P.dense(x, w, b, residual=r, activation=act), want["y"])
        leaves = [t.detach().requires_grad_() for t in (x, w, b, r) if t is not None]
        it = iter(leaves)
        xg, wg = next(it), next(it)
        bg, rg = next(it) if b is not None else None, next(it) if r is not None else None
        y = P.dense(xg, wg, bg, residual=rg, activation=act)
        close("y", y.detach(), want["y"])
        grads = torch.autograd.grad(y, leaves, dy)
        close("dx", grads[0], want["dx"])
        close("dw", grads[1], want["dw"])
        if b is not None:
            close("db", grads[2], want["db"])
        if r is not None:
            assert torch.equal(grads[-1], dy)
        again = torch.autograd.grad(P.dense(xg, wg, bg, residual=rg, activation=act), leaves, dy)
        assert all(torch.equal(p, q) for p, q in zip(grads, again))          # the same bits


@pytest.mark.parametrize("pad", [(1, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("size", [(5, 9, 7), (70, 130, 66), (1030, 70, 2050)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_nothing_around_strided_operands_is_used(pad, size, layout):
    import torch
    import paper_1710_06952_amd as P
    print(pad, size, layout, flush=True)
    x, w, b, r, dy = make(*size, torch.bfloat16, layout, seed=3, pad=pad)
    want = reference(x, w, b, r, dy, "silu")
    y, slope = P.dense_forward(x, w, b, residual=r, activation="silu")
    close("y", y, want["y"])
    for name, g in zip(("dx", "dw", "db"), P.dense_gradients(dy, x, w, slope, activation="silu")):
        close(name, g, want[name])


def test_values_that_are_not_finite_stay_in_their_rows():
    import torch
    import paper_1710_06952_amd as P
    x, w, b, r, dy = make(70, 33, 130, torch.bfloat16, "nk", seed=4)
    good, slope = P.dense_forward(x, w, b, residual=r, activation="gelu")
    dx = P.dense_gradients(dy, x, w, slope, activation="gelu")[0]
    bad_x, bad_dy = x.clone(), dy.clone()
    bad_x[17, 32] = math.inf
    bad_x[69, 0] = math.nan
    bad_dy[69] = math.nan
    y = P.dense(bad_x, w, b, residual=r, activation="gelu")
    rows = [i for i in range(70) if i not in (17, 69)]
    assert torch.equal(y[rows], good[rows]) and not torch.isfinite(y[17]).any() and torch.isnan(y[69]).all()
    bad = P.dense_gradients(bad_dy, x, w, slope, activation="gelu")[0]
    assert torch.equal(bad[:69], dx[:69]) and torch.isnan(bad[69]).all()
    y, slope = P.dense_forward(bad_x, w, b, activation="silu")
    bad = P.dense_gradients(dy, x, w, slope, activation="silu")[0]
    assert torch.isnan(bad[69]).all() and torch.isfinite(bad[:17]).all()


def test_no_rows_more_dimensions_and_expanded_gradients():
    import torch
    import paper_1710_06952_amd as P
    x, w, b, r, dy = make(24, 40, 56, torch.bfloat16, "nk", seed=5)
    none = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda:0", requires_grad=True)
    wg, bg = w.clone().requires_grad_(), b.clone().requires_grad_()
    y = P.dense(none, wg, bg, activation="relu")
    assert y.shape == (0, 56)
    dn, dw, db = torch.autograd.grad(y, [none, wg, bg], torch.empty_like(y))
    assert dn.shape == (0, 40) and not dw.any() and not db.any()
    y3 = P.dense(x.view(2, 3, 4, 40), w, b, residual=r.view(2, 3, 4, 56), activation="gelu")
    assert torch.equal(y3.view(24, 56), P.dense(x, w, b, residual=r, activation="gelu"))
    xg = x.clone().requires_grad_()
    P.dense(xg, wg, bg).sum().backward()                 # a gradient of stride 0
    ones = torch.ones_like(dy)
    want = reference(x, w, b, None, ones, "none")
    close("dx", xg.grad, want["dx"])
    close("db", bg.grad, want["db"])
    # shared weights: one leaf, two uses
    w2 = (torch.randn(40, 40, device="cuda:0") / 7).bfloat16().requires_grad_()
    h = P.dense(x, w2, activation="silu")
    y = P.dense(h, w2)
    d2, = torch.autograd.grad(y, [w2], torch.ones_like(y))
    second = P.dense_gradients(torch.ones_like(y), h.detach(), w2.detach(), None)
    first = P.dense_gradients(second[0], x, w2.detach(), P.dense_forward(x, w2.detach(), activation="silu")[1], activation="silu")
    assert torch.equal(d2, first[1] + second[1])


@pytest.mark.parametrize("act", ACTS[2:])
def test_gradients_against_differences(act):
    """dx, dw, db against central differences of the layer's formula in 64 bits."""
    import torch
    import paper_1710_06952_amd as P
    x, w, b, r, dy = make(6, 10, 12, torch.float16, "nk", seed=6)
    y, slope = P.dense_forward(x, w, b, residual=r, activation=act)
    grads = P.dense_gradients(dy, x, w, slope, activation=act)
    want = reference(x, w, b, r, dy, act)
    f = lambda x, w, b: float((activation(torch.mm(x, w.t().contiguous()) + b, act)[0] * dy.double()).sum())  # noqa: E731
    at = [x.double(), w.double(), b.double()]
    step = 1e-5
    for k, name in enumerate(("dx", "dw", "db")):
        flat = at[k].reshape(-1)
        for e in range(0, flat.numel(), 7):
            v = []
            for sign in (1, -1):
                moved = [t.clone() for t in at]
                moved[k].view(-1)[e] += sign * step
                v.append(f(*moved))
            diff = (v[0] - v[1]) / (2 * step)
            assert abs(diff - float(grads[k].reshape(-1)[e])) <= float(want[name][1].reshape(-1)[e]) + 1e-8 * (1 + abs(diff))


def test_capture_and_other_streams():
    import torch
    import paper_1710_06952_amd as P
    for size in ((64, 784, 1024), (3, 2100, 70)):
        x, w, b, r, dy = make(*size, torch.bfloat16, "kn", seed=7)
        side = torch.cuda.Stream()
        y, slope = P.dense_forward(x, w, b, residual=r, activation="gelu")
        want = [y, *P.dense_gradients(dy, x, w, slope, activation="gelu")]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            y, slope = P.dense_forward(x, w, b, residual=r, activation="gelu")
            got = [y, *P.dense_gradients(dy, x, w, slope, activation="gelu")]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, slope = P.dense_forward(x, w, b, residual=r, activation="gelu")
            got = [y, *P.dense_gradients(dy, x, w, slope, activation="gelu")]
        for k in range(3):
            x.mul_(0.5)
            graph.replay()
            torch.cuda.synchronize()
            replayed = [t.clone() for t in got]
            y, slope = P.dense_forward(x, w, b, residual=r, activation="gelu")
            want = [y, *P.dense_gradients(dy, x, w, slope, activation="gelu")]
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(replayed, want)), k


def test_capture_with_autograd_is_refused():
    import torch
    import paper_1710_06952_amd as P
    x, w, b, r, dy = make(8, 16, 24, torch.bfloat16, "nk", seed=8)
    wg = w.clone().requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="dense_forward"):
            P.dense(x, wg, b)
        y = P.dense(x, w, b)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, P.dense(x, w, b))


def test_forward_mode_is_refused():
    import torch
    import paper_1710_06952_amd as P
    from torch.autograd import forward_ad
    x, w, b, r, dy = make(8, 16, 24, torch.bfloat16, "nk", seed=9)
    t = torch.arange(8, device="cuda:0")
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        db = forward_ad.make_dual(b, torch.ones_like(b))
        for call in (lambda: P.dense(dual, w), lambda: P.dense(x, w, db), lambda: P.dense_forward(dual, w), lambda: P.token_log_probs(dual, t)):
            with pytest.raises(NotImplementedError, match="forward mode"):
                call()
        P.dense(x, w)
    with pytest.raises(Exception):
        torch.func.vmap(lambda q: P.dense(q, w))(x[None])
    with pytest.raises(Exception):
        torch.func.jvp(lambda q: P.dense(q, w), (x,), (torch.ones_like(x),))


def test_dimensions_of_one_and_far_rows():
    """The stride of a dimension of size 1 says nothing, and rows that lie further apart than the kernels reach are copied."""
    import torch
    import paper_1710_06952_amd as P
    K, N, far = 40, 24, (1 << 22) + 8
    x, w, b, r, dy = make(3, K, N, torch.bfloat16, "nk", seed=10)
    def apart(t):
        big = torch.full((t.shape[0], far), math.nan, dtype=t.dtype, device=t.device)
        big[:, :t.shape[1]] = t
        return big[:, :t.shape[1]]
    for rows in (1, 3):
        xs, rs, dys = x[:rows], r[:rows], dy[:rows]
        want, slope = P.dense_forward(xs, w, b, residual=rs, activation="silu")
        grads = P.dense_gradients(dys, xs, w, slope, activation="silu")
        got, slope = P.dense_forward(apart(xs), w, b, residual=apart(rs), activation="silu")
        assert torch.equal(got, want)
        assert all(torch.equal(p, q) for p, q in zip(P.dense_gradients(apart(dys), apart(xs), w, slope, activation="silu"), grads))
    want = P.dense(x, w, b)
    assert torch.equal(P.dense(x, apart(w), b), want) and torch.equal(P.dense(x, apart(w.t().contiguous()).t(), b), want)
    assert torch.equal(P.dense(x, apart(w[:1]), b[:1]), P.dense(x, w[:1], b[:1]))
    one = P.dense(x[:, :1], w[:, :1])
    assert torch.equal(P.dense(x[:, :1].contiguous(), apart(w[:, :1].t().contiguous()).t()), one)
    tokens = torch.tensor([5], device="cuda:0")
    assert torch.equal(P.token_log_probs(apart(x[:1]), tokens), P.token_log_probs(x[:1], tokens))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_values_far_from_0(act, dtype):
    """Products of one term, so z is exact.  y keeps its relative accuracy on both sides: 2.6e-6 of the fit, and of the exponential up to
    2^-23 of its exponent, 58 at z = -9."""
    import torch
    import paper_1710_06952_amd as P
    T = getattr(torch, dtype)
    z = torch.linspace(-9.0, 9.0, 2048, device="cuda:0").to(T)
    y = P.dense(torch.ones(1, 1, dtype=T, device="cuda:0"), z[:, None].contiguous(), activation=act)
    a = activation(z.double(), act)[0]
    tiny = 2.0 ** -25 if T == torch.float16 else 1e-38
    off = (y[0].double() - a).abs()
    assert (off <= 1.01 * half(T) * a.abs() + 1.2e-5 * a.abs() + tiny).all(), float((off / a.abs().clamp(min=1e-30)).max())


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_slopes_far_from_0(act, dtype):
    """Products of one term, so z is exact.  db is the slope where dy is 1: its root is kept in steps of 1 / 46000, half of which is 2.2e-5 of the
    root in the slope, and its square where nothing else is left; beside that 1.2e-5 as for y, and where terms cancel 2^-22."""
    import torch
    import paper_1710_06952_amd as P
    T = getattr(torch, dtype)
    z = torch.linspace(-9.0, 9.0, 2048, device="cuda:0").to(T)[:, None].contiguous()
    one = torch.ones(1, 1, dtype=T, device="cuda:0")
    y, slope = P.dense_forward(one, z, activation=act)
    s = activation(z[:, 0].double(), act)[1]
    db = P.dense_gradients(torch.ones_like(y), one, z, slope, activation=act)[2]
    tiny = 2.0 ** -25 if T == torch.float16 else 1e-38
    bound = 1.01 * half(T) * s.abs() + 1.01 * (1.2e-5 * s.abs() + 2.2e-5 * s.abs().sqrt()) + 1.2e-10 + tiny + torch.where(z[:, 0].abs() < 3, 2.0 ** -22, 0.0)
    if act == "relu":
        bound = torch.zeros_like(bound)                  # 0 and 1 are kept as they are
    off = (db.double() - s).abs()
    assert (off <= bound).all(), float((off / bound).max())


@pytest.mark.parametrize("size", [(8, 4096, 4104), (9, 4096, 4104), (9, 4096, 4096), (64, 4096, 4096), (64, 4104, 4096), (17, 72, 104), (17, 73, 101), (16, 73, 101),
                                  (5, 1032, 1001), (5, 1024, 1001), (30, 1032, 1032), (3, 1040, 16416), (3, 1040, 16448), (3, 1024, 16416)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_both_sides_of_few_rows(size, layout):
    """Sizes next to the lines between the kernel for few rows and the tiles."""
    import torch
    import paper_1710_06952_amd as P
    print(size, layout, flush=True)
    x, w, b, r, dy = make(*size, torch.float16, layout, seed=11)
    want = reference(x, w, b, r, dy, "silu")
    y, slope = P.dense_forward(x, w, b, residual=r, activation="silu")
    close("y", y, want["y"])
    for name, g in zip(("dx", "dw", "db"), P.dense_gradients(dy, x, w, slope, activation="silu")):
        close(name, g, want[name])
