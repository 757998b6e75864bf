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


def timed(call, times=3):
    import torch
    call()
    first, last = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    first.record()
    for _ in range(times):
        call()
    last.record()
    torch.cuda.synchronize()
    return first.elapsed_time(last) / times


@pytest.mark.parametrize("M,K,N", [(4096, 1024, 4096), (4097, 1023, 4097), (1500, 1024, 1500), (64, 1024, 8192)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gates_without_a_product(M, K, N, dtype):
    """One-hot rows of x beside weights of which half are 0: half of the gates are sums of zeros among ordinary ones.  They keep their slope of 0, and the call
    takes about what it takes with others (adding each of them again took 60 to 200 times as long; 10 is far from both)."""
    import torch
    import paper_1710_06952_amd as P
    t = getattr(torch, dtype)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(M + N)
    at = torch.randint(0, K, (M,), generator=gen, device="cuda:0")
    x = torch.nn.functional.one_hot(at, K).to(t)
    w = torch.randn(2 * N, K, generator=gen, device="cuda:0").to(t)
    w[:N][torch.rand(N, K, generator=gen, device="cuda:0") < 0.5] = 0
    h, slopes = P.gated_forward(x, w, activation="relu")
    gate, up = w[:N].t()[at], w[N:].t()[at]
    assert torch.equal(h, torch.where(gate > 0, gate.float() * up.float(), 0.0).to(t))
    dh = torch.ones(M, N, dtype=t, device="cuda:0")
    dx = P.gated_gradients(dh, x, w, slopes, need=(True, False, False))[0]
    dz = torch.cat([torch.where(gate > 0, up, 0.0), gate.clamp(min=0)], 1).double()
    want, size = torch.mm(dz, w.double()), torch.mm(dz.abs(), w.double().abs())
    half = torch.finfo(t).eps / 2
    # a slope is kept within 2^-10 (fp16: 2^-16), dz rounded once, 2 N products added in 32 bits
    assert ((dx.double() - want).abs() <= 1.01 * ((2.0 ** -10 if t is torch.bfloat16 else 2.0 ** -16) + half + (2 * N + 8) * 2.0 ** -24) * size + half * want.abs() + 2.0 ** -24).all()
    other = torch.randn(M, K, generator=gen, device="cuda:0").to(t)
    ordinary, zeros = timed(lambda: P.gated_forward(other, w, activation="silu")), timed(lambda: P.gated_forward(x, w, activation="relu"))
    assert zeros < 10 * ordinary + 0.2, "%.3f ms for %.3f" % (zeros, ordinary)


@pytest.mark.parametrize("M,K,N", [(64, 64, 1), (64, 64, 9), (16, 64, 17), (64, 32, 8), (64, 4000, 9)])
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_few_steps_of_a_column_alone(M, K, N, layout):
    """Where one wavefront has all the products of a column alone, its rows tell what is small: no more gates than those next to 0 are added again (all of them: 67 us
    for 6; four times the time of silu and 10 us are far from both)."""
    import torch
    import paper_1710_06952_amd as P
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(M + K + N)
    x, w = (torch.randn(*s, generator=gen, device="cuda:0").bfloat16() for s in ((M, K), (2 * N, K)))
    w = w if layout == "nk" else w.t().contiguous().t()
    graphs = []
    for act in ("silu", "relu"):
        P.gated_forward(x, w, activation=act)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for _ in range(50):
                P.gated_forward(x, w, activation=act)
    ordinary, corner = (timed(g.replay) / 50 for g in graphs)
    assert corner < 4 * ordinary + 0.01, "%.4f ms for %.4f" % (corner, ordinary)
