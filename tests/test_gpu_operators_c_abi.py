"""The operators of a worker's own training step from plain C and from several threads (GPU)."""
import os
import subprocess
import threading

import pytest

pytestmark = pytest.mark.gpu


def test_a_step_from_plain_c():
    """tests/c_abi/gpu_operators.c, built by __graft_entry__.build()."""
    exe = os.path.join(os.path.dirname(os.path.abspath(__file__)), "c_abi", "gpu_operators")
    if not os.path.exists(exe):          # one second of gcc, no GPU work
        import __graft_entry__
        exe = __graft_entry__.build_c_abi_program("gpu_operators")
    out = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert out.returncode == 0, (out.returncode, out.stdout, out.stderr)
    assert "c abi operators ok" in out.stdout


def test_two_threads_with_an_optimizer_each():
    """Each on a stream of its own, with its own refusals: the results are those of one after the other."""
    import torch
    import paper_1710_06952_amd as P

    def train(seed, bits):
        g = torch.Generator(device="cuda:0")
        g.manual_seed(seed)
        w, x = (torch.randn(*s, generator=g, device="cuda:0").bfloat16() for s in ((96, 80), (40, 80)))
        grad = torch.zeros_like(w)
        opt = P.AdamW([w], [grad], lr=1e-2, state_bits=bits, seed=seed)
        tokens = torch.arange(40, device="cuda:0")
        adv = torch.randn(40, generator=g, device="cuda:0")
        for _ in range(12):
            z = P.dense(x, w)
            r = P.policy_loss_and_gradient(z, tokens, P.token_log_probs(z, tokens), adv)
            grad.copy_(P.dense_gradients(r.dlogits, x, w, None, need=(False, True, False))[1])
            opt.step(max_norm=1.0)
            with pytest.raises(P.AdpsgdError, match="max_norm" if bits == 8 else "lr"):
                if bits == 8:
                    opt.step(max_norm=-1.0)
                else:
                    opt.lr = float("nan")
                    try:
                        opt.step()
                    finally:
                        opt.lr = 1e-2
        torch.cuda.current_stream().synchronize()
        return w, *opt.moments()
    want = [train(1, 32), train(2, 8)]
    torch.cuda.synchronize()
    got, faults = [None, None], []

    def run(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                got[k] = train(k + 1, (32, 8)[k])
                torch.cuda.current_stream().synchronize()
        except BaseException as e:      # noqa: B036  shown below
            faults.append(e)
    threads = [threading.Thread(target=run, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not faults and not any(t.is_alive() for t in threads), faults
    for p, q in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(p, q))
