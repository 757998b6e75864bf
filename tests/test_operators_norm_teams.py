"""Layer norm of fp32 rows against the formulas in 64 bits, with the additions that the lanes of a row's team do (GPU).

u = 2^-24.  On its way into a sum of a row a value passes L additions: those of a thread's elements, six steps over a wavefront and one for each wavefront of the team.  The
mean's first part m1 is off by f = (L + 2) u mean |x|;  c = x - m1 rounds once;  its mean m2 is off by (L + 2) u mean |c|, c - m2 and the product with r round once
each.  The sum of squares is off by (L + 2) u of itself, the instruction for 1 / sqrt by its last place, 2 u, so r by (L + 8) u / 2 + 2 u of itself and a little."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def additions(n, forward):
    """Of a row of n elements in fp32: vectors of four, and the elements behind the last whole vector one for each of the first lanes."""
    vectors = n // 4
    shapes = [(8, 8, 1), (16, 16, 1), (32, 32, 1), (64, 64, 1), (128, 64, 2)]
    shapes += [(256, 64, 4), (512, 256, 2), (1024, 256, 4), (2048, 1024, 2), (4096, 1024, 4)] if forward else [(256, 256, 1), (512, 512, 1), (1024, 1024, 1), (2048, 512, 4)]
    for most, lanes, held in shapes:
        if vectors <= most:
            return 4 * held + 1 + 6 + (lanes // 64 if lanes > 64 else 0)
    return 4 * -(-vectors // 1024) + 1 + 6 + 16


@pytest.mark.parametrize("n", [1, 7, 32, 61, 128, 257, 515, 1021, 1030, 2051, 4104, 8192, 8200, 16390, 32771, 70001])
@pytest.mark.parametrize("mean", [0.0, 0.5, 30.0])
def test_against_64_bits(n, mean):
    import torch
    import paper_1710_06952_amd as P
    rows, eps = 20, 1e-5
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(n)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda:0")  # noqa: E731
    x, w, b, dy = rand(rows, n) + mean, 1 + 0.3 * rand(n), 0.2 * rand(n), rand(rows, n)
    y, stats = P.layer_norm_forward(x, w, b, eps=eps)
    dx, dw, db = P.layer_norm_gradients(dy, x, w, stats)
    x, w, b, dy = (t.double() for t in (x, w, b, dy))
    avg = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    L, G = additions(n, True), additions(n, False)
    c = x - avg(x)
    s = torch.sqrt(avg(c * c) + eps)
    h = c / s
    first = (L + 2) * U * avg(x.abs())
    near = c.abs() + first
    dc = 2 * U * near + (L + 2) * U * avg(near) + U * first
    dr = ((L + 8) / 2 + 2) * U + avg(near * dc) / (s * s)
    dh = dc / s + h.abs() * (dr + 2 * U)

    def close(name, got, want, bound):
        off = float(((got.double() - want).abs() / (1.01 * bound + 1e-38)).max())
        assert off <= 1.0, "%s: %.3f of the bound" % (name, off)
    close("y", y, h * w + b, dh * w.abs() + 2 * U * ((h * w).abs() + b.abs()))
    g = dy * w
    A, B = avg(g), avg(g * h)
    dA = (G + 3) * U * avg(g.abs())
    dB = (G + 4) * U * avg((g * h).abs()) + avg(g.abs() * dh)
    size = g.abs() + A.abs() + (h * B).abs()
    close("dx", dx, (g - A - h * B) / s, (dA + dB * h.abs() + dh * B.abs() + size * (dr + 5 * U)) / s)
    dwant, dsize = (dy * h).sum(0), (dy * h).abs().sum(0)
    close("dw", dw, dwant, (dy.abs() * dh).sum(0) + (rows + 2) * U * dsize)
    close("db", db, dy.sum(0), (rows + 2) * U * dy.abs().sum(0))
