"""Gated projections (GPU): gradients from dz in two parts, the same gradients whatever else is asked for, and the same bits from the same inputs."""
import pytest

from test_operators_gated import half, make

pytestmark = pytest.mark.gpu


# dz has M 2 N elements: up to 4096 in the first six, a few over in the last two; dw has more than 8192 in all, dx in some
@pytest.mark.parametrize("M,K,N", [(3, 2224, 16), (1, 9000, 8), (2, 9, 1024), (1, 9, 2048), (7, 1300, 292), (128, 515, 16), (2, 9, 1025), (1, 9, 2049)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_gradients_from_few_elements_of_dz(M, K, N, dtype, layout):
    """With an activation of "none" a slope is the partner or the gate, a sum of K terms of 32 bits, kept within 2^-10 (fp16: 2^-16); dz in two parts is within half a
    step squared of itself, and a result's own rounding is half a step.  dz rounded once would be half a step more in every term."""
    import torch
    import paper_1710_06952_amd as P
    t = getattr(torch, dtype)
    x, w, b, dh = make(M, K, N, t, layout, 3 * M + K + N)
    _, slopes = P.gated_forward(x, w, b, activation="none")
    dx, dw, _ = P.gated_gradients(dh, x, w, slopes)
    f16, h, u = t is torch.float16, half(t), 2.0 ** -24
    x, w, dh, b = x.double(), w.double().contiguous(), dh.double(), b.double()
    z = torch.mm(x, w.t().contiguous()) + b
    zerr = (K + 8) * u * (torch.mm(x.abs(), w.abs().t().contiguous()) + b.abs())
    slope, off = torch.cat([z[:, N:], z[:, :N]], 1), torch.cat([zerr[:, N:], zerr[:, :N]], 1)
    d2 = torch.cat([dh, dh], 1)
    dz = d2 * slope
    off = d2.abs() * (off + (2.0 ** -16 if f16 else 2.0 ** -10) * (slope.abs() + off) + (1e-38 if f16 else 1e-14)) + 2 * u * dz.abs()
    parts = h * h if M * 2 * N <= 4096 else h
    err = off + 1.01 * parts * (dz.abs() + off) + (2.0 ** -25 if f16 else 0.0)
    mm = lambda p, q: torch.mm(p.contiguous(), q.contiguous())  # noqa: E731
    tiny = 2.0 ** -25 if f16 else 1e-30
    for name, got, want, terms, size in (("dx", dx, mm(dz, w), mm(err, w.abs()), mm(dz.abs(), w.abs())), ("dw", dw, mm(dz.t(), x), mm(err.t(), x.abs()), mm(dz.abs().t(), x.abs()))):
        inner = 4 * N if name == "dx" else 2 * M
        bound = 1.01 * (h * want.abs() + terms + (inner + 8) * u * size) + tiny
        worst = float(((got.double() - want).abs() / bound).max())
        assert worst <= 1.0, "%s: %.3f of the bound" % (name, worst)


# Products that copy operands to whole pieces, for both at once where dx and dw are asked for; neither dimension in whole pieces, and 2 N in them
@pytest.mark.parametrize("M,K,N", [(1101, 1021, 2001), (1101, 1021, 2004), (1203, 901, 2003)])
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_what_is_asked_for_changes_no_result(M, K, N, layout):
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dh = make(M, K, N, torch.bfloat16, layout, 7)
    _, slopes = P.gated_forward(x, w, b)
    full = P.gated_gradients(dh, x, w, slopes)
    for needed in ((True, False, False), (False, True, False), (False, False, True), (True, True, False), (True, False, True), (False, True, True)):
        for got, all3, asked in zip(P.gated_gradients(dh, x, w, slopes, need=needed), full, needed):
            assert torch.equal(got, all3) if asked else got is None


@pytest.mark.parametrize("M,K,N,dtype,layout,act", [(64, 784, 1024, "bfloat16", "kn", "gelu"), (2003, 1021, 2731, "float16", "nk", "relu"), (2048, 2048, 4096, "bfloat16", "nk", "silu"),
                                                    (256, 8192, 128, "bfloat16", "nk", "relu"), (1, 4096, 768, "float16", "kn", "silu")])
def test_the_same_bits_every_time(M, K, N, dtype, layout, act):
    """Sums have an order that the sizes give: beside other work, in other memory and from another stream too."""
    import torch
    import paper_1710_06952_amd as P
    x, w, b, dh = make(M, K, N, getattr(torch, dtype), layout, 8)
    side, first = torch.cuda.Stream(), None
    for turn in range(6):
        busy = torch.randn(256 + 1000 * turn, 1024, device="cuda:0")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side if turn % 2 else torch.cuda.current_stream()):
            h, slopes = P.gated_forward(x, w, b, activation=act)
            all4 = (h, *P.gated_gradients(dh, x, w, slopes))
        busy = busy * 2.0
        torch.cuda.synchronize()
        first = first or all4
        assert all(torch.equal(p, q) for p, q in zip(first, all4))
