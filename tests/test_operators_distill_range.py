"""The distillation loss of rows whose logits are far from 0 (GPU): only their differences matter."""
import pytest

pytestmark = pytest.mark.gpu


# Rows held by one wavefront and by blocks, few rows in two passes, one token, more entries than tokens, odd vocabularies
@pytest.mark.parametrize("rows,vocab,k", [(5, 1, 65), (5, 21, 1), (9, 176, 3), (40, 1001, 64), (200, 5000, 300), (3, 40_001, 70), (1, 131_072, 256)])
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("temperature,hard", [(1.0, 0.0), (1.5, 0.3), (7.0, 0.0)])
def test_far_from_0(rows, vocab, k, kind, temperature, hard):
    """Logits of one value next to 10^20 .. 10^38 of either sign, so q is 1 / vocab and KL = sum p log p + log vocab.  log vocab is within 1e-7 of itself (the sum of
    equal exponentials, its logarithm and their rounding to fp32), p log p within 3e-7 of the teacher's largest difference, and KL is rounded once."""
    import math
    import torch
    import paper_1710_06952_amd as P
    T = getattr(torch, kind)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(rows + vocab + k)
    size = torch.tensor([1e20, -3e25, 7e29, -2e33, 3e38], device="cuda:0").repeat(rows // 5 + 1)[:rows]
    z = size.to(T)[:, None].expand(rows, vocab).contiguous()
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda:0")
    entries = torch.randint(0, vocab, (rows, k), generator=gen, device="cuda:0")
    told = 3 * torch.randn(rows, k, generator=gen, device="cuda:0")
    r = P.distillation_loss_and_gradient(z, tokens, entries, told, temperature=temperature, hard_weight=hard)
    logp = torch.log_softmax(told.double() / temperature, 1)
    p = logp.exp()
    want = (p * logp).sum(1) + math.log(vocab)
    bound = 2e-7 * math.log(vocab) + 3e-7 * (logp.abs().amax(1) + 1) + 2.0 ** -24 * want.abs()
    assert ((r.divergences.double() - want).abs() <= bound).all()
    loss = ((1 - hard) * temperature ** 2 * want + hard * math.log(vocab)).mean()
    assert abs(float(r.loss) - float(loss)) <= temperature ** 2 * float(bound.max()) + 2e-7 * (abs(float(loss)) + math.log(vocab))
    onehot = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda:0").scatter_add_(1, entries, p)
    label = torch.nn.functional.one_hot(tokens, vocab).double()
    grad = ((1 - hard) * temperature * (1 / vocab - onehot) + hard * (1 / vocab - label)) / rows
    unit = ((1 - hard) * temperature + hard) / rows
    half = torch.finfo(T).eps / 2
    # 16 bits: half a step, and q within 1e-5 where its exponent is rounded beside z; q and p within 1e-6 else
    assert ((r.dlogits.double() - grad).abs() <= half * grad.abs() + unit * (1e-6 + 1e-5 / vocab)).all()


def test_beside_ordinary_logits():
    """One large logit with all of the teacher's weight: KL is 0 but for the teacher's own; with the weight on another, the distance."""
    import torch
    import paper_1710_06952_amd as P
    z = torch.randn(2, 300, device="cuda:0")
    z[:, 7] = 1e30
    tokens = torch.tensor([7, 7], device="cuda:0")
    r = P.distillation_loss_and_gradient(z, tokens, torch.tensor([[7, 7, -1], [9, 9, 9]], device="cuda:0"), torch.zeros(2, 3, device="cuda:0"), temperature=1.5)
    want = torch.tensor([0.0, (1e30 - float(z[1, 9])) / 1.5], dtype=torch.float64)
    # entries of the same token each with their own logarithm: -log 2 and -log 3
    own = torch.log(torch.tensor([2.0, 3.0], dtype=torch.float64))
    assert abs(float(r.divergences[0]) + float(own[0])) < 1e-6
    assert abs(float(r.divergences[1]) - float(want[1])) <= 2.0 ** -23 * float(want[1])
