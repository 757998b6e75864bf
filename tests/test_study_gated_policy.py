"""The policy study's normalised gated block and its distillation loss: the run and its gradients (GPU), not how far a loss falls."""
import numpy as np
import pytest

from paper_1710_06952_amd.studies import policy_model as S


def test_views_of_the_flat_vector():
    import torch
    p = S.Policy(11, 8, 5, 0, "cpu", "gated")
    x = torch.from_numpy(p.initial(0))
    assert x.numel() == p.d == 8 + 8 + 32 * 8 + 8 * 16 + 88 + 11
    parts = p.views(x)
    assert [tuple(v.shape) for v in parts] == p.shapes and torch.equal(torch.cat([v.reshape(-1) for v in parts]), x)
    assert (parts[0] == 1).all() and not parts[1].any()
    with pytest.raises(ValueError, match="block"):
        S.Policy(11, 8, 5, 0, "cpu", "round")


@pytest.mark.gpu
@pytest.mark.parametrize("loss,block", [("policy", "gated"), ("preference", "gated"), ("distill", "gated"), ("distill", "dense")])
def test_the_study_runs(loss, block):
    res = S.run_study(loss, n=4, vocab=72, width=64, prompts_each=16, M=48, events=48, gamma=5e-3, seed=1, block=block)
    assert res["events"] == 48 == sum(res["steps"]) and res["block"] == block
    assert np.isfinite(res["losses"]).all() and np.isfinite(res["chance"]).all() and np.isfinite(res["consensus_distance"])
    assert "quarter" in S.format_table(res)


@pytest.mark.gpu
@pytest.mark.parametrize("M,width,vocab", [(24, 64, 72), (7, 40, 33), (130, 136, 520)])
def test_gradients_of_the_whole_block(M, width, vocab):
    """layer_norm, gated, dense with the residual, dense and the distillation loss with their gradients, against autograd in 64 bits on the same bf16
    weights.  Six roundings to bf16 stand between a weight and the loss forward (norm, gated, block, logits and the block's own
    values again) and as many back: (2^-8 each relative to a tensor's size, in the mean over its elements a third of that) 5 % of each gradient's norm is over
    twice their sum, 12 2^-8 / 2 = 2.3 %."""
    import torch
    import paper_1710_06952_amd as P
    policy = S.Policy(vocab, width, 40, 3, "cuda:0", "gated")
    flat = torch.from_numpy(policy.initial(3)).cuda().bfloat16()
    leaves = [v.detach().clone().requires_grad_() for v in policy.views(flat)]
    asked = torch.arange(M, device="cuda:0") % 40
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(5)
    tokens = torch.randint(0, vocab, (M,), device="cuda:0", generator=gen)
    tokens[::5] = -1
    told = torch.randn(M, vocab, device="cuda:0", generator=gen)
    teacher = torch.topk(told, 6, 1)
    logits = policy.logits(leaves, asked)
    r = P.distillation_loss_and_gradient(logits, tokens, teacher.indices, teacher.values, temperature=2.0, hard_weight=0.25)
    grads = torch.autograd.grad(logits, leaves, r.dlogits)

    exact = [t.detach().double().cpu().requires_grad_() for t in leaves]
    scale, shift, wg, wd, w2, b2 = exact
    e = policy.embeddings[asked].double().cpu()
    g, u = (torch.nn.functional.layer_norm(e, (width,), scale, shift, 1e-5) @ wg.t()).chunk(2, 1)
    z = (torch.nn.functional.silu(g) * u @ wd.t() + e) @ w2.t() + b2
    counted = (tokens >= 0).cpu()
    log_p = torch.log_softmax(teacher.values.double().cpu() / 2.0, 1)
    log_q = torch.log_softmax(z / 2.0, 1).gather(1, teacher.indices.cpu())
    hard = -torch.log_softmax(z, 1).gather(1, tokens.clamp(min=0).cpu()[:, None])[:, 0]
    loss = (0.75 * 4.0 * (log_p.exp() * (log_p - log_q)).sum(1) + 0.25 * hard)[counted].mean()
    loss.backward()
    assert abs(float(r.loss) - float(loss)) < 0.03 * float(loss)
    for got, want in zip(grads, exact):
        off = float((got.double().cpu() - want.grad).norm() / want.grad.norm())
        assert off < 0.05, (tuple(want.shape), off)


@pytest.mark.gpu
def test_a_step_of_all_operators_captured():
    """The step as a captured graph: layer norm, gated, dense, the distillation loss and all gradients, replayed with new data and compared with the same calls."""
    import torch
    import paper_1710_06952_amd as P
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(9)
    new = lambda *s: torch.randn(*s, device="cuda:0", generator=gen)  # noqa: E731
    width, hidden, vocab, M = 64, 96, 200, 50
    scale, shift = (1 + 0.1 * new(width)).bfloat16(), (0.1 * new(width)).bfloat16()
    wg, wd, w2 = ((new(a, b) / b ** 0.5).bfloat16() for a, b in ((2 * hidden, width), (width, hidden), (vocab, width)))

    def step(e, tokens, entries, told):
        n, stats = P.layer_norm_forward(e, scale, shift)
        h, slopes = P.gated_forward(n, wg)
        r, _ = P.dense_forward(h, wd, residual=e)
        z, _ = P.dense_forward(r, w2)
        loss = P.distillation_loss_and_gradient(z, tokens, entries, told, temperature=2.0, hard_weight=0.1)
        dr, dw2, _ = P.dense_gradients(loss.dlogits, r, w2, None)
        dh, dwd, _ = P.dense_gradients(dr, h, wd, None)
        dn, dwg, _ = P.gated_gradients(dh, n, wg, slopes)
        de, ds, dt = P.layer_norm_gradients(dn, e, scale, stats)
        return loss.loss, z, dw2, dwd, dwg, ds, dt, de + dr

    def data():
        tokens = torch.randint(-20, vocab, (M,), device="cuda:0", generator=gen)
        top = torch.topk(new(M, vocab), 7, 1)
        return new(M, width).bfloat16(), tokens, top.indices, top.values

    held = data()
    step(*held)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*held)
    for _ in range(4):
        fresh = data()
        for to, x in zip(held, fresh):
            to.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(captured, step(*fresh)):
            assert torch.equal(got, want)
