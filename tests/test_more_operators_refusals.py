"""What layer norm, the gated projections and the distillation loss refuse, at the C entries (host checks, before anything touches a GPU) and in Python."""
import ctypes as C

import pytest

import paper_1710_06952_amd as P
from paper_1710_06952_amd import binding as B

NOWHERE = 1 << 20                                        # an aligned address that is never read


def refused(rc, word):
    assert rc == B.ERR_ARG
    assert word in B.lib().adpsgd_last_error(None).decode(), B.lib().adpsgd_last_error(None)


def norm_args(**kw):
    o = dict(type=B.TYPE_BF16, param_type=B.TYPE_BF16, rows=4, n=16, x=NOWHERE, ldx=16, w=NOWHERE, b=NOWHERE, eps=1e-5, workspace=NOWHERE,
             workspace_bytes=1 << 20)
    o.update(kw)
    return B.LayerNorm(**o)


@pytest.mark.parametrize("change,word", [
    (dict(type=5), "type"), (dict(param_type=B.TYPE_F16), "type"), (dict(type=B.TYPE_F32), "type"), (dict(rows=-1), "rows"), (dict(n=0), "rows"), (dict(n=(1 << 28) + 1, ldx=1 << 29), "rows"),
    (dict(rows=(1 << 31) + 1), "rows"), (dict(rows=1 << 30, n=1 << 20, ldx=1 << 20), "rows"), (dict(ldx=15), "leading"), (dict(ldx=1 << 41), "leading"), (dict(x=None), "NULL"),
    (dict(w=None), "without w"), (dict(x=NOWHERE + 1), "aligned"), (dict(w=NOWHERE + 1), "aligned"), (dict(param_type=B.TYPE_F32, b=NOWHERE + 2), "aligned")])
def test_layer_norm(change, word):
    L = B.lib()
    refused(L.adpsgd_layer_norm_forward(C.byref(norm_args(**change)), NOWHERE, NOWHERE, None), word)
    refused(L.adpsgd_layer_norm_backward(C.byref(norm_args(**change)), NOWHERE, 1 << 20, NOWHERE, NOWHERE, NOWHERE, NOWHERE, None), word)


def test_layer_norm_calls():
    L, at = B.lib(), NOWHERE
    refused(L.adpsgd_layer_norm_forward(None, at, at, None), "no arguments")
    for eps in (0.0, -1e-5, 1e-40, float("inf"), float("nan")):
        refused(L.adpsgd_layer_norm_forward(C.byref(norm_args(eps=eps)), at, at, None), "eps")
    refused(L.adpsgd_layer_norm_forward(C.byref(norm_args()), None, at, None), "y is NULL")
    refused(L.adpsgd_layer_norm_forward(C.byref(norm_args()), at + 1, at, None), "aligned")
    refused(L.adpsgd_layer_norm_forward(C.byref(norm_args()), at, at + 2, None), "aligned")
    o = norm_args()
    refused(L.adpsgd_layer_norm_backward(C.byref(o), None, 16, at, at, at, at, None), "dy or stats")
    refused(L.adpsgd_layer_norm_backward(C.byref(o), at, 16, None, at, at, at, None), "dy or stats")
    refused(L.adpsgd_layer_norm_backward(C.byref(o), at, 15, at, at, at, at, None), "leading dimension of dy")
    refused(L.adpsgd_layer_norm_backward(C.byref(norm_args(w=None, b=None)), at, 16, at, at, at, None, None), "dw without w")
    refused(L.adpsgd_layer_norm_backward(C.byref(o), at, 16, at, at, at + 1, at, None), "aligned")
    for short in (dict(workspace_bytes=8), dict(workspace=None), dict(workspace=at + 8)):
        refused(L.adpsgd_layer_norm_backward(C.byref(norm_args(rows=4000, **short)), at, 16, at, None, at, None, None), "workspace")
    assert L.adpsgd_layer_norm_forward(C.byref(norm_args(rows=0, x=None)), None, None, None) == B.OK       # no rows: nothing to do
    assert L.adpsgd_layer_norm_backward(C.byref(norm_args(rows=0, x=None)), None, 16, None, None, None, None, None) == B.OK
    assert L.adpsgd_layer_norm_workspace_bytes(9, 4, 16) == L.adpsgd_layer_norm_workspace_bytes(0, -1, 16) == L.adpsgd_layer_norm_workspace_bytes(0, 4, 0) == -1
    assert L.adpsgd_layer_norm_workspace_bytes(0, 0, 16) == 0 and L.adpsgd_layer_norm_workspace_bytes(1, 4000, 16) >= 256


def test_layer_norm_tensors_that_are_not_on_a_gpu():
    import torch
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for call in (lambda: P.layer_norm(x, w), lambda: P.layer_norm_forward(x, w, w), lambda: P.layer_norm_gradients(x, x, w, torch.zeros(3, 4))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError, match="tensor"):
        P.layer_norm([1.0])
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError, match="forward mode"):
            P.layer_norm(forward_ad.make_dual(x, x), w)


@pytest.mark.gpu
def test_layer_norm_shapes_and_types():
    import torch
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda:0")  # noqa: E731
    x, w, stats = new(4, 8), new(8), new(3, 4, dtype=torch.float32)
    for call, kind, word in [
            (lambda: P.layer_norm(x.double()), TypeError, "float32"), (lambda: P.layer_norm(x, w.half()), TypeError, "both"), (lambda: P.layer_norm(x.float(), w), TypeError, "both"),
            (lambda: P.layer_norm(x, w, w.float()), TypeError, "both"), (lambda: P.layer_norm(x, None, w), ValueError, "without a weight"),
            (lambda: P.layer_norm(x, new(7)), ValueError, "weight is"), (lambda: P.layer_norm(x, w, new(1, 8)), ValueError, "bias is"), (lambda: P.layer_norm(x, w.cpu()), ValueError, "GPU"),
            (lambda: P.layer_norm(new(4, 0)), ValueError, "last dimension"), (lambda: P.layer_norm(x, eps=0.0), P.AdpsgdError, "eps"),
            (lambda: P.layer_norm_gradients(x.float(), x, w, stats), ValueError, "dy is"), (lambda: P.layer_norm_gradients(x[:3], x, w, stats), ValueError, "dy is"),
            (lambda: P.layer_norm_gradients(x, x, w, stats[:, :3]), ValueError, "stats"), (lambda: P.layer_norm_gradients(x, x, w, stats.half()), ValueError, "stats")]:
        with pytest.raises(kind, match=word):
            call()


def gated_args(**kw):
    o = dict(type=B.TYPE_BF16, activation=B.ACT_SILU, M=4, N=8, K=16, x=NOWHERE, ldx=16, w=NOWHERE, ldw=16, w_transposed=0, workspace=NOWHERE,
             workspace_bytes=1 << 30)
    o.update(kw)
    return B.Dense(**o)


@pytest.mark.parametrize("change,word", [
    (dict(type=B.TYPE_F32), "type"), (dict(activation=9), "activation"), (dict(M=-1), "M >= 0"), (dict(N=0), "M >= 0"), (dict(K=0), "M >= 0"), (dict(N=1 << 62), "M >= 0"),
    (dict(ldx=15), "leading"), (dict(ldw=15), "leading"), (dict(w_transposed=1, ldw=15), "leading"), (dict(r=NOWHERE, ldr=8), "residual"), (dict(ldx=(1 << 22) + 1), "2^22"),
    (dict(N=(1 << 21) + 1), "2^22"), (dict(M=1 << 30, N=1 << 10), "2^34"), (dict(x=None), "NULL"), (dict(w=None), "NULL"), (dict(x=NOWHERE + 1), "aligned"),
    (dict(b=NOWHERE + 1), "aligned")])
def test_gated(change, word):
    L = B.lib()
    refused(L.adpsgd_gated_forward(C.byref(gated_args(**change)), NOWHERE, None, None), word)
    refused(L.adpsgd_gated_backward(C.byref(gated_args(**change)), NOWHERE, 1 << 22, NOWHERE, NOWHERE, NOWHERE, NOWHERE, None), word)


def test_gated_calls():
    L, at = B.lib(), NOWHERE
    refused(L.adpsgd_gated_forward(None, at, None, None), "no arguments")
    refused(L.adpsgd_gated_forward(C.byref(gated_args()), None, None, None), "h is NULL")
    refused(L.adpsgd_gated_forward(C.byref(gated_args()), at, at + 1, None), "aligned")
    refused(L.adpsgd_gated_backward(C.byref(gated_args()), at, 8, None, at, None, None, None), "slopes")
    refused(L.adpsgd_gated_backward(C.byref(gated_args()), None, 8, at, at, None, None, None), "dh")
    refused(L.adpsgd_gated_backward(C.byref(gated_args()), at, 7, at, at, None, None, None), "leading dimension of dh")
    refused(L.adpsgd_gated_backward(C.byref(gated_args()), at, 8, at, at + 1, None, None, None), "aligned")
    for short in (dict(workspace_bytes=8), dict(workspace=None), dict(workspace=at + 4)):
        refused(L.adpsgd_gated_backward(C.byref(gated_args(**short)), at, 8, at, at, None, None, None), "workspace")
    refused(L.adpsgd_gated_forward(C.byref(gated_args(K=1 << 13, ldx=1 << 13, ldw=1 << 13, workspace_bytes=8)), at, None, None), "workspace")
    assert L.adpsgd_gated_forward(C.byref(gated_args(M=0, x=None)), None, None, None) == B.OK        # no rows: nothing to do
    assert L.adpsgd_gated_backward(C.byref(gated_args()), at, 8, at, None, None, None, None) == B.OK       # nothing asked for
    for sizes in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1 << 20, 1 << 20, 1), (1, 1 << 62, 1)):
        assert L.adpsgd_gated_workspace_bytes(*sizes, 0) == -1 and L.adpsgd_gated_workspace_bytes(*sizes, 1) == -1
    assert L.adpsgd_gated_workspace_bytes(64, 1024, 784, 1) >= 4 * 64 * 1024
    assert L.adpsgd_gated_slopes_bytes(B.TYPE_BF16, 3, 5) == 60 and L.adpsgd_gated_slopes_bytes(B.TYPE_F16, 3, 5) == 90
    assert L.adpsgd_gated_slopes_bytes(B.TYPE_F32, 3, 5) == L.adpsgd_gated_slopes_bytes(B.TYPE_F16, -1, 5) == L.adpsgd_gated_slopes_bytes(B.TYPE_F16, 1, 0) == -1


def test_gated_tensors_that_are_not_on_a_gpu():
    import torch
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(6, 8, dtype=torch.bfloat16)
    for call in (lambda: P.gated(x, w), lambda: P.gated_forward(x, w), lambda: P.gated_gradients(x[:, :3], x, w, torch.zeros(48, dtype=torch.uint8))):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError, match="tensor"):
        P.gated([1.0], w)
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError, match="forward mode"):
            P.gated(forward_ad.make_dual(x, x), w)


@pytest.mark.gpu
def test_gated_shapes_and_types():
    import torch
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda:0")  # noqa: E731
    x, w, dh, slopes = new(4, 8), new(6, 8), new(4, 3), new(48, dtype=torch.uint8)
    for call, kind, word in [
            (lambda: P.gated(x, new(6, 9)), ValueError, "2 out x in"), (lambda: P.gated(x, new(5, 8)), ValueError, "2 out x in"), (lambda: P.gated(x, new(0, 8)), ValueError, "2 out x in"),
            (lambda: P.gated(x.float(), w.float()), TypeError, "float32"), (lambda: P.gated(x, w.half()), TypeError, "float16"), (lambda: P.gated(x, w, new(3)), ValueError, "bias"),
            (lambda: P.gated(x, w, activation="tanh"), ValueError, "activation"), (lambda: P.gated(x, w.cpu()), ValueError, "GPU"),
            (lambda: P.gated_gradients(new(4, 6), x, w, slopes), ValueError, "dh is"), (lambda: P.gated_gradients(dh.half(), x, w, slopes), ValueError, "dh is"),
            (lambda: P.gated_gradients(dh, x, w, slopes[:47]), ValueError, "slopes"), (lambda: P.gated_gradients(dh, x, w, slopes.half()), ValueError, "slopes")]:
        with pytest.raises(kind, match=word):
            call()


def logits_args(**kw):
    o = dict(type=B.TYPE_BF16, rows=4, vocab=100, z=NOWHERE, ld=100, tokens=NOWHERE, workspace=NOWHERE, workspace_bytes=1 << 20)
    o.update(kw)
    return B.Logits(**o)


def teacher_args(**kw):
    o = dict(type=B.TYPE_F32, k=8, tokens=NOWHERE, ld_tokens=8, z=NOWHERE, ld=8)
    o.update(kw)
    return B.Teacher(**o)


def distill(o=None, t=None, T=1.0, a=0.0, scale=1.0, loss=NOWHERE, dz=NOWHERE, kl=NOWHERE, logp=None):
    return B.lib().adpsgd_distillation_loss(C.byref(o or logits_args()), C.byref(t or teacher_args()), T, a, scale, loss, dz, kl, logp, None)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(rows=-1), "rows"), (dict(vocab=0), "rows"), (dict(ld=99), "leading"), (dict(z=None), "NULL"), (dict(tokens=None), "NULL"),
    (dict(tokens=NOWHERE + 4), "aligned"), (dict(workspace=None), "workspace"), (dict(workspace=NOWHERE + 8), "workspace"), (dict(workspace_bytes=4 * 9 * 8), "workspace")])
def test_distillation_logits(change, word):
    refused(distill(logits_args(**change)), word)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(k=0), "1024"), (dict(k=1025), "1024"), (dict(ld=7), "leading"), (dict(ld_tokens=7), "leading"), (dict(ld=1 << 41), "leading"), (dict(z=None), "NULL"),
    (dict(tokens=None), "NULL"), (dict(tokens=NOWHERE + 4), "aligned"), (dict(z=NOWHERE + 2), "aligned")])
def test_distillation_teacher(change, word):
    refused(distill(t=teacher_args(**change)), word)


def test_distillation_calls():
    L, at = B.lib(), NOWHERE
    refused(L.adpsgd_distillation_loss(None, C.byref(teacher_args()), 1.0, 0.0, 1.0, at, at, at, None, None), "no arguments")
    refused(L.adpsgd_distillation_loss(C.byref(logits_args()), None, 1.0, 0.0, 1.0, at, at, at, None, None), "no teacher")
    for T in (0.0, -1.0, 1e-7, 1e7, float("nan"), float("inf")):
        refused(distill(T=T), "temperature")
    for a in (-0.1, 1.0, float("nan")):
        refused(distill(a=a, logp=at), "hard_weight")
    for scale in (float("inf"), float("nan"), 1e30):
        refused(distill(scale=scale), "loss_scale")
    refused(distill(a=0.1), "log_probs")
    refused(distill(logp=at), "log_probs")
    for kw in (dict(loss=None), dict(dz=None), dict(kl=None)):
        refused(distill(**kw), "NULL")
    for kw in (dict(loss=at + 2), dict(dz=at + 1), dict(kl=at + 2), dict(a=0.1, logp=at + 2)):
        refused(distill(**kw), "aligned")
    W = L.adpsgd_distillation_workspace_bytes
    assert W(-1, 10, 1) == W(1, 0, 1) == W(1, 10, 0) == W(1, 10, 1025) == -1 and W(100, 10, 16) >= 100 * 17 * 8 and W(0, 10, 1) > 0


def test_distillation_tensors_that_are_not_on_a_gpu():
    import torch
    z, tokens = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        P.distillation_loss_and_gradient(z, tokens, tokens[:, None], z[:, :1])
    with pytest.raises(TypeError, match="tensor"):
        P.distillation_loss_and_gradient([1.0], tokens, tokens[:, None], z[:, :1])
    from torch.autograd import forward_ad
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError, match="forward mode"):
            P.distillation_loss_and_gradient(forward_ad.make_dual(z, z), tokens, tokens[:, None], z[:, :1])


@pytest.mark.gpu
def test_distillation_shapes_and_types():
    import torch
    new = lambda *s, dtype=torch.int64: torch.zeros(*s, dtype=dtype, device="cuda:0")  # noqa: E731
    z, tokens, e, t = new(4, 8, dtype=torch.float32), new(4), new(4, 2), new(4, 2, dtype=torch.float32)
    call = P.distillation_loss_and_gradient
    for run, kind, word in [
            (lambda: call(z.double(), tokens, e, t), TypeError, "logits"), (lambda: call(z[0], tokens, e, t), ValueError, "rows"), (lambda: call(z, tokens[:3], e, t), ValueError, "tokens"),
            (lambda: call(z, tokens, e[:3], t), ValueError, "teacher_tokens"), (lambda: call(z, tokens, e, t[:3]), ValueError, "teacher_logits"),
            (lambda: call(z, tokens, e[:, :0], t), ValueError, "teacher_tokens"), (lambda: call(z, tokens, e, t[:, :1]), TypeError, "same shape"),
            (lambda: call(z, tokens, e.int(), t), TypeError, "int64"), (lambda: call(z, tokens, e, t.double()), TypeError, "float32"), (lambda: call(z, tokens, e.cpu(), t), ValueError, "GPU"),
            (lambda: call(z, tokens, new(4, 1025), new(4, 1025, dtype=torch.float32)), P.AdpsgdError, "1024"), (lambda: call(z, tokens, e, t, temperature=0.0), P.AdpsgdError, "temperature"),
            (lambda: call(z, tokens, e, t, hard_weight=1.5), P.AdpsgdError, "hard_weight"), (lambda: call(z, tokens, e, t, loss_scale=float("nan")), P.AdpsgdError, "loss_scale")]:
        with pytest.raises(kind, match=word):
            run()


@pytest.mark.parametrize("name", ["_LayerNorm", "_Gated"])
def test_a_captured_backward_pass(name, monkeypatch):
    """Refused before it looks at anything, on the CPU with the capture made up."""
    import torch
    from paper_1710_06952_amd import operators
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="captured"):
        getattr(operators, name).backward(object(), torch.zeros(1))


@pytest.mark.gpu
def test_a_captured_backward_pass_of_eager_graphs():
    """... and in a capture on the stream of the forward pass, behind which the same graphs give their gradients."""
    import torch
    new = lambda *s: torch.randn(*s, device="cuda:0").bfloat16()  # noqa: E731
    side = torch.cuda.Stream()
    x, w, b, wg, dy = new(24, 64).requires_grad_(), new(64), new(64), new(80, 64), new(24, 64)
    dh = new(24, 40)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y, h = P.layer_norm(x, w, b), P.gated(x, wg)
    for out, d, word in ((y, dy, "layer_norm"), (h, dh, "gated")):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side), pytest.raises(RuntimeError, match=word):
            torch.autograd.grad(out, x, d, retain_graph=True)
    torch.cuda.synchronize()
    _, stats = P.layer_norm_forward(x.detach(), w, b)
    _, slopes = P.gated_forward(x.detach(), wg)
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], P.layer_norm_gradients(dy, x.detach(), w, stats)[0])
    assert torch.equal(torch.autograd.grad(h, x, dh)[0], P.gated_gradients(dh, x.detach(), wg, slopes)[0])
