"""Layer norm of finite rows next to the ends of their type (GPU): rows of one large value, and rows whose spread is more than the largest number."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def half(t):
    import torch
    return torch.finfo(t).eps / 2


# Rows held by every team of lanes, forward and backward, with elements behind the last vector, and rows in passes
@pytest.mark.parametrize("n", [1, 4, 16, 300, 768, 1000, 1024, 3000, 5000, 9001, 20000, 40000])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("eps", [1e-5, 2.0 ** -120])
def test_rows_of_one_large_value(kind, n, eps):
    """x - mean is 0 whatever the sums round to: y = b and dw = 0 exactly, and dx = (g - mean g) / sqrt(eps).

    dx: r is one rounding and the instruction's last place (2 u), g = dy w one, the mean at most n + 2 of mean |g|, the difference and the product
    one each, and the type's: 6 u (|g| + mean |g|) / sqrt(eps) + (n + 2) u mean |g| / sqrt(eps) + half a step."""
    import torch
    import paper_1710_06952_amd as P
    T = getattr(torch, kind)
    least, most = torch.finfo(T).min, torch.finfo(T).max
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(n)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda:0")  # noqa: E731
    values = torch.tensor([2e38, -1e30, 1e35, least, most, 1e26, 1e24, -1e20, 0.0], device="cuda:0")
    x = values.to(T)[:, None].expand(-1, n).contiguous()
    assert torch.isfinite(x).all()
    w, b, dy = 1 + 0.3 * rand(n), 0.2 * rand(n), rand(len(values), n).to(T)
    y, stats = P.layer_norm_forward(x, w, b, eps=eps)
    assert torch.isfinite(stats).all()
    assert torch.equal(y, b.to(T).expand_as(y))
    assert torch.equal(P.layer_norm(x, w, b, eps=eps), y)
    dx, dw, db = P.layer_norm_gradients(dy, x, w, stats)
    assert not dw.any()
    r = 1 / math.sqrt(eps)
    g = dy.double() * w.double()
    mean, size = g.mean(1, keepdim=True), g.abs().mean(1, keepdim=True)
    want = r * (g - mean)
    bound = half(T) * want.abs() + 1.01 * r * U * (6 * (g.abs() + size) + (n + 2) * size) + 1e-38
    assert ((dx.double() - want).abs() <= bound).all()
    total = dy.double().sum(0)
    assert ((db.double() - total).abs() <= 20 * U * dy.double().abs().sum(0)).all()


@pytest.mark.parametrize("n", [2, 7, 16, 300, 1000, 2051, 5000, 9001, 20000, 40000])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_rows_whose_spread_is_more_than_the_largest_number(kind, n):
    """Values up to the ends of the type, among them some more than the largest number away from the mean.

    c = x - mean is off by u (2 |c| + (L + 4) X) with X the largest |c| and L <= n / 8 + 16 additions on a value's way into a sum, 1 / s by (L + 8) u of itself, and
    behind the forward pass by half a step of the subnormal numbers, which is 2^-150 s of itself."""
    import torch
    import paper_1710_06952_amd as P
    T = getattr(torch, kind)
    most = torch.finfo(T).max
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(n + 1)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda:0")  # noqa: E731
    share = torch.rand(4, n, generator=gen, device="cuda:0") * 0.3 - 0.9
    share[:, 0], share[2:, n // 2] = 0.98, 1.0
    share[3] = -share[3]
    x = (share.double() * most).to(T)
    assert torch.isfinite(x).all()
    w, b, dy = 1 + 0.3 * rand(n), 0.2 * rand(n), (2.0 ** 20 * rand(4, n)).to(T)          # dx of 2^-106, not of 2^-126
    y, stats = P.layer_norm_forward(x, w, b)
    assert torch.isfinite(stats).all()
    xd, d = x.double(), dy.double()
    c = xd - xd.mean(1, keepdim=True)
    if n > 4:
        assert float(c.abs().max()) > torch.finfo(torch.float32).max
    s = (c * c).mean(1, keepdim=True).sqrt()
    h, X, L = c / s, c.abs().amax(1, keepdim=True), n / 8 + 16
    off = U * (2 * c.abs() + (L + 4) * (X + xd.abs().mean(1, keepdim=True))) / s + h.abs() * (L + 8) * U
    want = h * w + b
    assert ((y.double() - want).abs() <= half(T) * want.abs() + 1.01 * (off * w.abs() + 3 * U * ((h * w).abs() + b.abs())) + 1e-38).all()
    dx, dw, db = P.layer_norm_gradients(dy, x, w, stats)
    off = off + h.abs() * 2.0 ** -150 * s
    want = (d * h).sum(0)
    assert ((dw.double() - want).abs() <= 1.01 * (U * want.abs() + (d.abs() * off).sum(0) + 12 * U * (d * h).abs().sum(0))).all()
    assert ((db.double() - d.sum(0)).abs() <= 12 * U * d.abs().sum(0)).all()
    g = d * w.double()
    A, B = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    size, want = (g.abs() + A.abs() + (h * B).abs()) / s, (g - A - h * B) / s
    bound = half(T) * want.abs() + size * ((3 * L + 40) * U + 2.0 ** -150 * s) + ((g.abs() * off).mean(1, keepdim=True) * h.abs() + off * B.abs()) / s
    assert ((dx.double() - want).abs() <= 1.01 * bound + 1e-38).all()
