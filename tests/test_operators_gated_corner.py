"""Gated projections with relu: gates next to 0 (GPU).  A sum in 32 bits has either sign there; the slope is the one of the sum in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


def rows_next_to_the_corner(M, K, N, column, every, t, seed):
    """x and w of type t with the gates of `column` within a few 2^-24 of their terms' sum of 0 in every `every`-th row, and those rows' sums in 64 bits: their last
    inputs take away what the sum of the others comes to, two roundings deep in fp16 (2^-11 each) and three in bf16 (2^-8 each)."""
    import torch
    gen = torch.Generator()
    gen.manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen).to(t)  # noqa: E731
    depth = 2 if t is torch.float16 else 3
    x, w = new(M, K), new(2 * N, K)
    rows = torch.arange(every - 1, M, every)
    for d in range(depth):
        w[column, K - depth + d] = 2.0 ** (-8 * d)
    x[rows, K - depth:] = 0
    rest = x[rows].double() @ w[column].double()
    for d in range(depth):
        scale = 2.0 ** (-8 * d)
        x[rows, K - depth + d] = (-rest / scale).to(t)
        rest = rest + x[rows, K - depth + d].double() * scale
    return x, w, rows, rest


# The column is alone in its eight: one column, or the last one of 8 n + 1.  One row, few rows, tiles of 64, 128 and 256, sums of parts, copies of whole pieces
@pytest.mark.parametrize("M,K,N", [(1, 500, 1), (9, 500, 9), (40, 1000, 1), (60, 4100, 17), (300, 1000, 1), (300, 1000, 9), (1100, 200, 1001), (256, 8192, 129), (2050, 72, 2049), (2100, 1030, 2049)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_a_column_alone(M, K, N, dtype, layout):
    """dh is 1 in the column, so dx of a row is u times the gate's weights where the gate is over 0 (and next to nothing of the partner's: act(g) is under 1e-4), and 0 else."""
    import torch
    import paper_1710_06952_amd as P
    t = getattr(torch, dtype)
    x, w, rows, rest = rows_next_to_the_corner(M, K, N, N - 1, min(M, 8), t, M + K + N)
    wd = w.cuda() if layout == "nk" else w.t().contiguous().cuda().t()
    _, slopes = P.gated_forward(x.cuda(), wd, activation="relu")
    dh = torch.zeros(M, N, dtype=t)
    dh[:, N - 1] = 1
    dx = P.gated_gradients(dh.cuda(), x.cuda(), wd, slopes, need=(True, False, False))[0].cpu().double()[rows]
    partner = x[rows].double() @ w[2 * N - 1].double()
    wg = w[N - 1].double()
    share = (dx @ wg) / (wg @ wg)                        # of the gate's weights in dx: the partner or 0
    sure = (partner.abs() > 1e-2) & (rest.abs() > 1e-12)
    wrong = ((share.abs() > 0.5 * partner.abs()) != (rest > 0)) & sure
    assert not wrong.any(), "%d of %d on the other side" % (int(wrong.sum()), int(sure.sum()))
