"""Layer norm, gated projections and the distillation loss from plain C and from several threads (GPU)."""
import os
import subprocess
import threading

import pytest

pytestmark = pytest.mark.gpu


def test_a_step_from_plain_c():
    """tests/c_abi/gpu_more_operators.c, built by __graft_entry__.build()."""
    exe = os.path.join(os.path.dirname(os.path.abspath(__file__)), "c_abi", "gpu_more_operators")
    if not os.path.exists(exe):          # one second of gcc, no GPU work
        import __graft_entry__
        exe = __graft_entry__.build_c_abi_program("gpu_more_operators")
    out = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert out.returncode == 0, (out.returncode, out.stdout, out.stderr)
    assert "c abi more operators ok" in out.stdout


def test_two_threads():
    """Each on a stream of its own, with refusals between: the results are those of one after the other."""
    import torch
    import paper_1710_06952_amd as P

    def steps(seed):
        g = torch.Generator(device="cuda:0")
        g.manual_seed(seed)
        new = lambda *s: torch.randn(*s, generator=g, device="cuda:0").bfloat16()  # noqa: E731
        x, scale, w, out = new(200, 72), new(72), new(128, 72) * 0.1, new(300, 64) * 0.1
        tokens = torch.arange(200, device="cuda:0")
        got = []
        for turn in range(10):
            n, stats = P.layer_norm_forward(x, scale)
            h, slopes = P.gated_forward(n, w, activation="gelu")
            z = P.dense(h, out)
            top = torch.topk(z.float(), 9, 1)
            r = P.distillation_loss_and_gradient(z, tokens, top.indices, top.values + turn, temperature=1.5, hard_weight=0.3)
            dh = P.dense_gradients(r.dlogits, h, out, None, need=(True, False, False))[0]
            dn, dw, _ = P.gated_gradients(dh, n, w, slopes)
            dx, ds, _ = P.layer_norm_gradients(dn, x, scale, stats)
            with pytest.raises(P.AdpsgdError, match="temperature" if seed == 1 else "eps"):
                if seed == 1:
                    P.distillation_loss_and_gradient(z, tokens, top.indices, top.values, temperature=-1.0)
                else:
                    P.layer_norm(x, scale, eps=-1.0)
            x = (x.float() - 100.0 * dx.float()).bfloat16()
            got += [r.loss, z, dw, ds]
        torch.cuda.current_stream().synchronize()
        return got
    want = [steps(1), steps(2)]
    torch.cuda.synchronize()
    got, faults = [None, None], []

    def run(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                got[k] = steps(k + 1)
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
