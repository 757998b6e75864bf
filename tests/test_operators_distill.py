"""The distillation loss and its gradient against the formulas in 64 bits (GPU).

Tolerances.  u = 2^-24.  A sum of exponentials of a row is off by E = (160 + 3 D) u of itself: up to 128 terms of a thread one after the other and 16
joins, and each exponential by its argument's two roundings and the instruction's own 2 u, D = the largest |z - m| / T log2 e that has weight (its
terms under e^-30 have none; 45).  KL is off by E + 40 u max |log p| + what its double precision loses, nothing.  A gradient's element is
cs q_T: q_T by E + (3 D(z) + 8) u where D(z) is that element's own, an entry's p by 16 u; one rounding to the type."""
import math

import pytest

pytestmark = pytest.mark.gpu

# (rows, vocab, k): one of everything, less than a vector, every block of the kernel that holds rows, in passes, few rows, the most entries
SIZES = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 33, 33), (70, 100, 5), (64, 1000, 8), (9, 2049, 64), (33, 4100, 65), (40, 9001, 50), (6, 20000, 100), (35, 33333, 7),
         (40, 50001, 50), (34, 65540, 256), (33, 131080, 16), (3, 131072, 256), (2, 150001, 1024), (1100, 600, 300), (2, 5000, 1024), (2500, 40, 4), (50, 1500, 1023)]
KINDS = [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("bfloat16", "float16")]


def half(t):
    import torch
    return torch.finfo(t).eps / 2


def make(rows, vocab, k, kind, teacher, seed, pad=0, masked=0.2, spread=2.5):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda:0")  # noqa: E731
    store = torch.full((rows, vocab + pad), math.nan, dtype=getattr(torch, kind), device="cuda:0")
    z = store[:, :vocab]
    z.copy_(spread * rand(rows, vocab))
    top = torch.topk(z.float() + rand(rows, vocab), min(k, vocab), 1)
    entries, t = top.indices, top.values
    if k > vocab:                                            # tokens that come again
        more = torch.randint(0, vocab, (rows, k - vocab), generator=g, device="cuda:0")
        entries, t = torch.cat([entries, more], 1), torch.cat([t, rand(rows, k - vocab)], 1)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda:0")
    tokens = torch.where(torch.rand(rows, generator=g, device="cuda:0") < masked, -1 - tokens, tokens)
    return z, tokens, entries.contiguous(), t.to(getattr(torch, teacher)).contiguous()


def reference(z, tokens, entries, t, T, a, scale=1.0):
    """loss, dlogits, divergences, log_probs with the bounds of all but the first."""
    import torch
    u, D = 2.0 ** -24, 45.0
    E = (160 + 3 * D) * u
    R, V = z.shape
    h = half(z.dtype)
    tiny = 2.0 ** -25 if z.dtype == torch.float16 else 1e-37
    counted = tokens >= 0
    n = max(1, int(counted.sum()))
    zd, td = z.double(), t.double()
    used = entries >= 0
    log_qT, log_q = torch.log_softmax(zd / T, 1), torch.log_softmax(zd, 1)
    some = used.any(1, keepdim=True)
    log_p = torch.log_softmax((td / T).masked_fill(~used, -math.inf), 1)
    p = torch.where(used & some, log_p.exp(), 0.0)
    at = entries.clamp(min=0)
    terms = torch.where(p > 0, p * (log_p - log_qT.gather(1, at)), 0.0)
    kl = torch.where(counted, terms.sum(1), 0.0)
    dkl = torch.where(counted, E + 40 * u * torch.where(p > 0, log_p.abs() + 1, 0.0).amax(1) + 2 * u * kl.abs(), 0.0)
    hot = tokens.clamp(min=0)[:, None]
    logp = torch.where(counted, log_q.gather(1, hot)[:, 0], 0.0)
    dlogp = torch.where(counted, E + 4 * u * logp.abs(), 0.0)
    cs = (counted[:, None] & some).double() * (scale * (1 - a) * T / n)
    ch = counted[:, None].double() * (scale * a / n)
    off = lambda l: l.exp() * (E + (3 * l.clamp(min=-200).abs() * 1.45 + 12) * u)  # noqa: E731
    d = cs * log_qT.exp() + ch * log_q.exp()
    bound = cs.abs() * off(log_qT) + ch.abs() * off(log_q)
    weight = torch.zeros_like(d).scatter_add_(1, at, p)
    d = d - cs * weight
    bound = bound + 16 * u * cs.abs() * weight
    d.scatter_add_(1, hot, -ch)
    bound.scatter_add_(1, hot, 4 * u * ch.abs())
    loss = float(((1 - a) * T * T * kl - a * logp).sum() / n)
    dloss = float(((1 - a) * T * T * dkl + a * dlogp).sum() / n) + 4 * u * abs(loss)
    return dict(loss=(loss, dloss), dlogits=(d, 1.01 * h * d.abs() + 1.01 * bound + tiny), divergences=(kl, dkl + 1e-37), log_probs=(logp, dlogp + 1e-37))


def close(name, got, want):
    import torch
    value, bound = want
    off = (got.double() - value).abs()
    assert got.shape == value.shape and torch.isfinite(got).all(), name
    worst = float((off / bound).max()) if off.numel() else 0.0
    assert worst <= 1.0, "%s: %.3f of the bound" % (name, worst)


def check(r, want, hard):
    assert abs(float(r.loss) - want["loss"][0]) <= want["loss"][1], (float(r.loss), want["loss"])
    close("dlogits", r.dlogits, want["dlogits"])
    close("divergences", r.divergences, want["divergences"])
    if hard:
        close("log_probs", r.log_probs, want["log_probs"])
    else:
        assert r.log_probs is None


def same(r, q):
    import torch
    return all((a is None and b is None) or torch.equal(a, b) for a, b in zip(r, q))


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind,teacher", KINDS)
def test_loss_and_gradient(size, kind, teacher):
    import paper_1710_06952_amd as P
    scale = 64.0 * size[0] if kind == "float16" else 1.0
    for T, a in ((1.0, 0.0), (2.0, 0.0), (1.5, 0.3), (1.0, 0.5)):
        z, tokens, entries, t = make(*size, kind, teacher, size[0] * 31 + size[1] + size[2], pad=3)
        r = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=T, hard_weight=a, loss_scale=scale)
        assert r.dlogits.dtype == z.dtype
        check(r, reference(z, tokens, entries, t, T, a, scale), a)


@pytest.mark.parametrize("vocab", [50, 1000, 30000, 140000])
def test_entries_that_are_not_there_and_rows_that_are_empty(vocab):
    import torch
    import paper_1710_06952_amd as P
    z, tokens, entries, t = make(40, vocab, 12, "float32", "float32", 3, masked=0.1)
    tokens[:8] = torch.arange(8, device="cuda:0")
    entries[0] = -1                                          # no entry at all
    entries[1, 3:] = -5                                      # three
    entries[2, ::2] = -1
    t[3, 1:] = -math.inf                                     # one with weight
    entries[4, :] = 7                                        # all the same token
    entries[5, 4:8] = entries[5, 0:4]                        # some twice
    tokens[6] = entries[6, 2]                                # the token is an entry
    t[7] = torch.finfo(torch.float32).min                    # the lowest value everywhere: uniform
    z[20:] = z[20:].clone().index_fill_(1, torch.arange(vocab - 5, vocab, device="cuda:0"), -math.inf)
    gone = (entries[20:] >= vocab - 5) | (tokens[20:, None] >= vocab - 5)
    entries[20:] = torch.where(gone, 1, entries[20:])
    tokens[20:] = torch.where(tokens[20:] >= vocab - 5, 1, tokens[20:])
    for T, a in ((1.0, 0.0), (3.0, 0.0), (2.0, 0.2)):
        want = reference(z, tokens, entries, t, T, a)
        r = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=T, hard_weight=a)
        check(r, want, a)
        assert r.divergences[0] == 0 and (a > 0 or not r.dlogits[0].any())
        assert not r.dlogits[tokens < 0].any()
    again = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=2.0, hard_weight=0.2)
    assert same(r, again)


@pytest.mark.parametrize("vocab", [40, 3000, 140000])
def test_what_has_no_number(vocab):
    """NaN and infinities stay in their rows; tokens beyond the vocabulary are never followed."""
    import torch
    import paper_1710_06952_amd as P
    z, tokens, entries, t = make(12, vocab, 6, "bfloat16", "float32", 4, masked=0.0)
    good = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=2.0, hard_weight=0.1)
    z, tokens, entries, t = z.clone(), tokens.clone(), entries.clone(), t.clone()
    z[1, 5] = math.nan
    z[2] = -math.inf
    entries[3, 2] = vocab
    entries[4, 0] = 1 << 40
    t[5, 1] = math.nan
    t[6] = -math.inf
    tokens[7] = vocab + 3
    z[8, 3] = math.inf
    tokens[9] = -1
    z[9] = math.nan                                          # not read
    entries[9] = 1 << 50
    r = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=2.0, hard_weight=0.1)
    share = 12 / 11
    assert r.loss.isnan() and not r.dlogits[9].any() and r.divergences[9] == 0
    assert r.divergences[[1, 2, 3, 4, 5, 6, 8]].isnan().all()
    for row in (1, 2, 3, 4, 5, 6, 7, 8):
        assert r.dlogits[row].isnan().all(), row
    for row in (0, 10, 11):
        off = (r.dlogits[row].double() - share * good.dlogits[row].double()).abs()
        assert (off <= share * 2.0 ** -8 * 2.1 * good.dlogits[row].double().abs()).all()
        assert r.divergences[row] == good.divergences[row]
    # an entry with weight that the student cannot say: an infinite loss, a finite gradient
    z, tokens, entries, t = make(4, vocab, 6, "float32", "float32", 5, masked=0.0)
    z[1, entries[1, 0]] = -math.inf
    tokens[1] = entries[1, 1]
    r = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=1.0, hard_weight=0.1)
    assert r.loss == math.inf and r.divergences[1] == math.inf and torch.isfinite(r.dlogits).all()
    assert r.dlogits[1, entries[1, 0]] < 0


def test_no_rows_and_no_counted_rows():
    import torch
    import paper_1710_06952_amd as P
    z, tokens, entries, t = make(5, 100, 4, "float32", "float32", 6)
    r = P.distillation_loss_and_gradient(z[:0], tokens[:0], entries[:0], t[:0])
    assert r.loss == 0 and r.dlogits.shape == (0, 100) and r.divergences.shape == (0,)
    r = P.distillation_loss_and_gradient(z, torch.full_like(tokens, -1), entries, t, hard_weight=0.5)
    assert r.loss == 0 and not r.dlogits.any() and not r.log_probs.any()


@pytest.mark.parametrize("vocab", [300, 40000, 140000])
def test_strides(vocab):
    import torch
    import paper_1710_06952_amd as P
    z, tokens, entries, t = make(33, vocab, 9, "bfloat16", "bfloat16", 7)
    want = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=2.0)
    zp = torch.full((35, vocab + 9), math.nan, dtype=z.dtype, device="cuda:0")
    zp[1:34, 4:4 + vocab] = z
    ep, tp = torch.full((33, 20), 1 << 45, device="cuda:0"), torch.full((33, 13), math.nan, dtype=t.dtype, device="cuda:0")
    ep[:, 5:14], tp[:, 1:10] = entries, t
    two = torch.stack([tokens, tokens + 5], 1)[:, 0]
    r = P.distillation_loss_and_gradient(zp[1:34, 4:4 + vocab], two, ep[:, 5:14], tp[:, 1:10], temperature=2.0)
    assert same(r, want)                                     # rows are cut where those of the gradient are
    r = P.distillation_loss_and_gradient(z, tokens, entries.t().contiguous().t(), t.t().contiguous().t(), temperature=2.0)
    assert same(r, want)


@pytest.mark.parametrize("T", [2.0 ** -10, 0.01, 0.3, 1.0, 7.0, 1000.0])
def test_temperatures(T):
    import paper_1710_06952_amd as P
    z, tokens, entries, t = make(20, 700, 20, "float32", "float32", 8, spread=max(1.0, min(T, 50.0)) if T > 0.1 else 4 * T)
    z = z.contiguous()
    if T < 0.1:
        t = t * (4 * T)
    for a in (0.0, 0.4):
        check(P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=T, hard_weight=a), reference(z, tokens, entries, t, T, a), a)


def test_against_differences():
    import paper_1710_06952_amd as P
    z, tokens, entries, t = make(6, 30, 5, "float32", "float32", 9)
    T, a = 2.0, 0.3
    r = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=T, hard_weight=a, loss_scale=3.0)
    for row in range(6):
        for v in (0, 11, int(entries[row, 0]), int(tokens[row].clamp(min=0))):
            plus, minus = z.double().clone(), z.double().clone()
            plus[row, v] += 1e-4
            minus[row, v] -= 1e-4
            slope = 3.0 * (reference(plus.float().double(), tokens, entries, t, T, a)["loss"][0]
                           - reference(minus.float().double(), tokens, entries, t, T, a)["loss"][0]) / float(plus.float()[row, v].double() - minus.float()[row, v].double())
            assert abs(slope - float(r.dlogits[row, v])) < 1e-6 + 1e-5 * abs(slope)


@pytest.mark.parametrize("size", [(64, 1000, 8), (8, 131072, 256), (1200, 2000, 16)], ids=str)
def test_another_stream_and_a_graph(size):
    import torch
    import paper_1710_06952_amd as P
    call = lambda *s: P.distillation_loss_and_gradient(*s, temperature=2.0, hard_weight=0.1)  # noqa: E731
    held = make(*size, "bfloat16", "bfloat16", 10)
    want = call(*held)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(*held)
    torch.cuda.current_stream().wait_stream(side)
    assert same(got, want)
    held = tuple(x.clone() for x in held)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call(*held)
    for turn in range(4):
        new = make(*size, "bfloat16", "bfloat16", 20 + turn)
        for to, x in zip(held, new):
            to.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert same(captured, call(*new))


@pytest.mark.parametrize("T,a", [(1.0, 0.0), (2.0, 0.0), (1.0, 0.25), (1.5, 0.25)])
@pytest.mark.parametrize("rows,vocab,k", [(64, 1000, 4), (1, 872, 2), (4, 5, 3), (3, 33333, 16), (1, 131072, 64), (100, 50001, 8), (17, 9001, 1), (2, 2049, 1024)])
def test_rows_that_are_sure_of_the_teachers_token(rows, vocab, k, T, a):
    """fp32 rows and teachers with nearly all weight on the same token: q - p is what two numbers next to 1 leave, 1 - q down to 10^-7.  An entry's q is e / (e + rest)
    with e to 10^-15 and the rest of the row off by E of itself, so q by E q (1 - q); its p by 3 u p (1 - p), each exponential rounded once.  What multiplies
    them and the rounding of the result are 6 u of it."""
    import torch
    import paper_1710_06952_amd as P
    z, _, _, _ = make(rows, vocab, 1, "float32", "float32", 31 + rows + k, masked=0.0)
    z = z.contiguous()
    tokens = torch.arange(rows, device="cuda:0") * 37 % vocab
    z[torch.arange(rows), tokens] += T * torch.linspace(9.0, 25.0, rows, device="cuda:0")
    g = torch.Generator(device="cuda:0")
    g.manual_seed(5)
    top = torch.topk(z + torch.randn(rows, vocab, generator=g, device="cuda:0"), k, 1)
    entries, t = top.indices.contiguous(), top.values.contiguous()
    got = P.distillation_loss_and_gradient(z, tokens, entries, t, temperature=T, hard_weight=a).dlogits.double()
    u = 2.0 ** -24
    E = (160 + 3 * 45) * u
    q, q1, p = torch.softmax(z.double() / T, 1), torch.softmax(z.double(), 1), torch.zeros(rows, vocab, dtype=torch.float64, device="cuda:0")
    p.scatter_(1, entries, torch.softmax(t.double() / T, 1))
    hot = torch.zeros_like(p).scatter_(1, tokens[:, None], 1.0)
    cs, ch = (1 - a) * T / rows, a / rows
    d = cs * (q - p) + ch * (q1 - hot)
    bound = cs * (E * q * (1 - q) + 3 * u * p * (1 - p)) + ch * E * q1 * (1 - q1) + 6 * u * (cs * (q - p).abs() + ch * (q1 - hot).abs()) + 1e-37
    apart = (p == 0) & (hot == 0)                            # an element of the pass: q by E as it is, and what it is multiplied with
    bound = torch.where(apart, (E + 60 * u) * (cs * q + ch * q1) + 1e-37, bound)
    assert ((got - d).abs() <= bound).all(), float(((got - d).abs() / bound).max())
