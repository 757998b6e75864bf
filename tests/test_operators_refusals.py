"""What the operators of a worker's training step refuse, at the C entries (host checks, before anything touches a GPU) and in Python."""
import ctypes as C

import numpy as np
import pytest

import paper_1710_06952_amd as P
from paper_1710_06952_amd import binding as B

NOWHERE = 1 << 20                                        # an aligned address that is never read


def refused(rc, word):
    assert rc == B.ERR_ARG
    assert word in B.lib().adpsgd_last_error(None).decode(), B.lib().adpsgd_last_error(None)


def dense_args(**kw):
    o = dict(type=B.TYPE_BF16, activation=B.ACT_GELU, M=4, N=8, K=16, x=NOWHERE, ldx=16, w=NOWHERE, ldw=16, w_transposed=0, workspace=NOWHERE,
             workspace_bytes=1 << 30)
    o.update(kw)
    return B.Dense(**o)


@pytest.mark.parametrize("change,word", [
    (dict(type=B.TYPE_F32), "type"), (dict(type=7), "type"), (dict(activation=9), "activation"), (dict(M=-1), "M >= 0"), (dict(N=0), "M >= 0"), (dict(K=0), "M >= 0"),
    (dict(ldx=15), "leading"), (dict(ldw=15), "leading"), (dict(w_transposed=1, ldw=7), "leading"), (dict(r=NOWHERE, ldr=7), "leading"),
    (dict(ldx=(1 << 22) + 1), "2^22"), (dict(M=1 << 30, N=1 << 10), "2^34"), (dict(x=None), "NULL"), (dict(w=None), "NULL"), (dict(x=NOWHERE + 1), "aligned"),
    (dict(b=NOWHERE + 1), "aligned")])
def test_dense(change, word):
    L = B.lib()
    refused(L.adpsgd_dense_forward(C.byref(dense_args(**change)), NOWHERE, None, None), word)
    refused(L.adpsgd_dense_backward(C.byref(dense_args(**change)), NOWHERE, 1 << 14, NOWHERE, NOWHERE, NOWHERE, NOWHERE, None), word)


def test_dense_calls():
    L = B.lib()
    refused(L.adpsgd_dense_forward(None, NOWHERE, None, None), "no arguments")
    refused(L.adpsgd_dense_forward(C.byref(dense_args()), None, None, None), "y is NULL")
    refused(L.adpsgd_dense_backward(C.byref(dense_args()), NOWHERE, 8, None, NOWHERE, None, None, None), "slopes")
    refused(L.adpsgd_dense_backward(C.byref(dense_args()), NOWHERE, 7, NOWHERE, NOWHERE, None, None, None), "dy")
    refused(L.adpsgd_dense_backward(C.byref(dense_args()), None, 8, NOWHERE, NOWHERE, None, None, None), "dy is NULL")
    refused(L.adpsgd_dense_backward(C.byref(dense_args(workspace_bytes=8)), NOWHERE, 8, NOWHERE, NOWHERE, None, None, None), "workspace")
    refused(L.adpsgd_dense_backward(C.byref(dense_args(workspace=NOWHERE + 4)), NOWHERE, 8, NOWHERE, NOWHERE, None, None, None), "workspace")
    assert L.adpsgd_dense_forward(C.byref(dense_args(M=0, x=None)), None, None, None) == B.OK        # no rows: nothing to do
    for sizes in ((-1, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1 << 20, 1 << 20, 1)):
        assert L.adpsgd_dense_workspace_bytes(*sizes, 0) == -1 and L.adpsgd_dense_workspace_bytes(*sizes, 1) == -1
    assert L.adpsgd_dense_workspace_bytes(64, 1024, 784, 1) >= 2 * 64 * 1024


def logits_args(**kw):
    o = dict(type=B.TYPE_BF16, rows=4, vocab=100, z=NOWHERE, ld=100, tokens=NOWHERE, workspace=NOWHERE, workspace_bytes=1 << 20)
    o.update(kw)
    return B.Logits(**o)


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(rows=-1), "rows"), (dict(vocab=0), "rows"), (dict(rows=1 << 21, vocab=1 << 20, ld=1 << 20), "rows"), (dict(ld=99), "leading"),
    (dict(z=None), "NULL"), (dict(tokens=None), "NULL"), (dict(tokens=NOWHERE + 4), "aligned"), (dict(type=B.TYPE_F32, z=NOWHERE + 2), "aligned"),
    (dict(workspace=None), "workspace"), (dict(workspace=NOWHERE + 8), "workspace"), (dict(workspace_bytes=16), "workspace")])
def test_logits(change, word):
    L, o = B.lib(), logits_args(**change)
    refused(L.adpsgd_token_log_probs(C.byref(o), NOWHERE, None), word)
    refused(L.adpsgd_policy_loss(C.byref(o), NOWHERE, NOWHERE, None, 0.2, 0.2, 0.0, NOWHERE, NOWHERE, NOWHERE, None), word)
    refused(L.adpsgd_preference_loss(C.byref(o), NOWHERE, 1, NOWHERE, 0.1, 0.0, NOWHERE, NOWHERE, NOWHERE, NOWHERE, None), word)


def test_losses():
    L, o = B.lib(), logits_args()
    at = NOWHERE
    refused(L.adpsgd_token_log_probs(C.byref(o), None, None), "log_probs")
    for lo, hi in ((-0.1, 0.2), (1.1, 0.2), (0.2, -0.1), (0.2, float("inf")), (float("nan"), 0.2)):
        refused(L.adpsgd_policy_loss(C.byref(o), at, at, None, lo, hi, 0.0, at, at, at, None), "clip")
    refused(L.adpsgd_policy_loss(C.byref(o), at, at, None, 0.2, 0.2, 0.1, at, at, at, None), "ref_log_probs")
    refused(L.adpsgd_policy_loss(C.byref(o), at, at, at, 0.2, 0.2, -0.1, at, at, at, None), "kl_coef")
    refused(L.adpsgd_policy_loss(C.byref(o), at, None, None, 0.2, 0.2, 0.0, at, at, at, None), "NULL")
    refused(L.adpsgd_policy_loss(C.byref(o), at, at, None, 0.2, 0.2, 0.0, None, at, at, None), "NULL")
    refused(L.adpsgd_policy_loss(C.byref(o), at + 2, at, None, 0.2, 0.2, 0.0, at, at, at, None), "aligned")
    refused(L.adpsgd_preference_loss(C.byref(o), at, 0, at, 0.1, 0.0, at, at, at, at, None), "pairs")
    refused(L.adpsgd_preference_loss(C.byref(o), at, 1, at, 0.0, 0.0, at, at, at, at, None), "beta")
    refused(L.adpsgd_preference_loss(C.byref(o), at, 1, at, 0.1, 0.5, at, at, at, at, None), "label_smoothing")
    refused(L.adpsgd_preference_loss(C.byref(o), None, 1, at, 0.1, 0.0, at, at, at, at, None), "NULL")
    refused(L.adpsgd_preference_loss(C.byref(o), at + 4, 1, at, 0.1, 0.0, at, at, at, at, None), "aligned")
    assert L.adpsgd_loss_workspace_bytes(-1, 10) == -1 and L.adpsgd_loss_workspace_bytes(1 << 22, 10) == -1 and L.adpsgd_loss_workspace_bytes(0, 10) > 0


def adamw_args(n=2, **kw):
    sizes = (C.c_int64 * n)(*[10] * n)
    pointers = (C.c_void_p * n)(*[NOWHERE] * n)
    decay = (C.c_float * n)(*[0.1] * n)
    o = dict(tensors=n, param_type=B.TYPE_BF16, grad_type=B.TYPE_BF16, state_bits=32, sizes=sizes, params=pointers, grads=pointers, masters=None, out=None,
             weight_decay=decay, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, m=NOWHERE, v=NOWHERE, exponents=None)
    o.update(kw)
    return B.AdamwOpts(**o)


@pytest.mark.parametrize("change,word", [
    (dict(param_type=5), "type"), (dict(state_bits=16), "state_bits"), (dict(beta1=1.0), "beta"), (dict(beta2=-0.1), "beta"), (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"),
    (dict(sizes=(C.c_int64 * 2)(10, -1)), "size"), (dict(params=None), "NULL"), (dict(params=(C.c_void_p * 2)(NOWHERE, None)), "NULL"),
    (dict(masters=(C.c_void_p * 2)(NOWHERE, None)), "NULL"), (dict(grads=(C.c_void_p * 2)(NOWHERE, NOWHERE + 1)), "aligned"), (dict(m=None), "m or v"), (dict(v=NOWHERE + 8), "m or v"),
    (dict(state_bits=8), "exponents"), (dict(weight_decay=(C.c_float * 2)(0.0, float("nan"))), "weight_decay")])
def test_adamw(change, word):
    h = C.c_void_p(1)
    refused(B.lib().adpsgd_adamw_create(C.byref(h), C.byref(adamw_args(**change))), word)
    assert not h.value


def test_adamw_calls():
    L = B.lib()
    refused(L.adpsgd_adamw_create(None, C.byref(adamw_args())), "no arguments")
    refused(L.adpsgd_adamw_step(None, 1e-3, 0.0, 1.0, None, None), "no handle")
    refused(L.adpsgd_adamw_get_moments(None, NOWHERE, NOWHERE, None), "no handle")
    assert L.adpsgd_adamw_get_steps(None, None) == B.ERR_ARG and L.adpsgd_adamw_set_steps(None, 1) == B.ERR_ARG
    assert L.adpsgd_adamw_state_length((C.c_int64 * 3)(1, 256, 257), 3) == 256 + 256 + 512
    assert L.adpsgd_adamw_state_length((C.c_int64 * 1)(-1), 1) == -1
    L.adpsgd_adamw_destroy(None)


def test_tensors_that_are_not_on_a_gpu():
    import torch
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        P.dense(x, w)
    with pytest.raises(ValueError, match="GPU"):
        P.token_log_probs(x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="GPU"):
        P.policy_loss_and_gradient(x, torch.zeros(4, dtype=torch.int64), x[:, 0], x[:, 0])
    with pytest.raises(ValueError, match="GPU"):
        P.AdamW([x], [x])
    with pytest.raises(TypeError, match="tensor"):
        P.dense(np.zeros((4, 8)), w)
    with pytest.raises(ValueError, match="lists"):
        P.AdamW([], [])
    with pytest.raises(AttributeError):
        P.no_such_operator


@pytest.mark.gpu
def test_shapes_and_types():
    import torch
    new = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda:0")  # noqa: E731
    x, w = new(4, 8), new(3, 8)
    for call, kind, word in [
            (lambda: P.dense(x, new(3, 9)), ValueError, "out x in"), (lambda: P.dense(x.float(), w.float()), TypeError, "float32"), (lambda: P.dense(x, w.half()), TypeError, "float16"),
            (lambda: P.dense(x, w, new(4)), ValueError, "bias"), (lambda: P.dense(x, w, residual=new(3)), ValueError, "residual"),
            (lambda: P.dense(x, w, activation="tanh"), ValueError, "activation"), (lambda: P.dense(x, w.cpu()), ValueError, "GPU"),
            (lambda: P.dense_gradients(new(4, 3), x, w, None, activation="relu"), TypeError, "slope"),
            (lambda: P.dense_gradients(new(4, 3), x, w, new(4, 3), activation="relu"), ValueError, "slope"),
            (lambda: P.token_log_probs(x, new(4)), ValueError, "tokens"), (lambda: P.token_log_probs(x.double(), new(4, dtype=torch.int64)), TypeError, "logits"),
            (lambda: P.token_log_probs(x[0], new(8, dtype=torch.int64)), ValueError, "vocabulary"),
            (lambda: P.policy_loss_and_gradient(x, new(4, dtype=torch.int64), new(4), new(4)), ValueError, "old_log_probs"),
            (lambda: P.preference_loss_and_gradient(x, new(4, dtype=torch.int64), new(4, dtype=torch.int64), new(2, dtype=torch.float32)), ValueError, "offsets"),
            (lambda: P.preference_loss_and_gradient(x, new(4, dtype=torch.int64), new(3, dtype=torch.int64), new(3, dtype=torch.float32)), ValueError, "ref_log_probs"),
            (lambda: P.AdamW([x], [w]), ValueError, "elements"), (lambda: P.AdamW([x, w.half()], [x, w]), TypeError, "same"), (lambda: P.AdamW([x.t()], [x.t()]), ValueError, "contiguous"),
            (lambda: P.AdamW([x], [x], masters=[x]), TypeError, "float32"), (lambda: P.AdamW([x], [x], state_bits=4), ValueError, "state_bits")]:
        with pytest.raises(kind, match=word):
            call()
    opt = P.AdamW([x], [x])
    with pytest.raises(P.AdpsgdError):
        opt.step(max_norm=-1.0)
    with pytest.raises(ValueError, match="steps"):
        opt.load_moments(new(256), new(256), -1)
    assert opt.steps == 0


def test_an_eps_that_is_no_normal_number():
    h = C.c_void_p(1)
    refused(B.lib().adpsgd_adamw_create(C.byref(h), C.byref(adamw_args(eps=1e-40))), "eps")
    assert not h.value


def test_an_optimizer_that_outlives_the_module(monkeypatch):
    """At the interpreter's end the module's names are None, and a collected optimizer says nothing."""
    from paper_1710_06952_amd import operators
    opt = operators.AdamW.__new__(operators.AdamW)
    opt._h = C.c_void_p(NOWHERE)
    monkeypatch.setattr(operators, "B", None)
    opt.close()
    assert opt._h is None


def test_forward_mode():
    import torch
    from torch.autograd import forward_ad
    x, w, t = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for call in (lambda: P.dense(dual, w), lambda: P.dense_forward(dual, w), lambda: P.token_log_probs(dual, t), lambda: P.AdamW([dual], [x]),
                     lambda: P.policy_loss_and_gradient(dual, t, x[:, 0], x[:, 0])):
            with pytest.raises(NotImplementedError, match="forward mode"):
                call()
        with pytest.raises(ValueError, match="GPU"):
            P.dense(x, w)
