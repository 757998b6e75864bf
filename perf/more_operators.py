"""More operators of a worker's own training step, as cases that can be timed and compared: layer norm, the gated first
half of a feed-forward block, and the distillation loss from a teacher's top logits.

A case names an operator and its sizes; ``prepare`` makes what a program holds before the call, ``run`` is one call:
through the framework's entry points where ``own`` is true, and else in plain torch operations in 32 bits (64 for sums
over rows and for what cancels).  ``exact`` is the same result from the operator's definition in 64 bits.

ops   norm     y = (x - mean) / sqrt(var + eps) w + b over rows, and with train dx, dw, db for a given dy
      gated    h = act(x Wg^T + bg) (x Wu^T + bu), w = [Wg; Wu], and with train dx, dw, db for a given dh
      distill  (1 - a) T^2 KL(teacher's top entries || softmax(z / T)) - a log softmax(z)[token], a mean over the rows
               that count, and the gradient of loss_scale times that for the logits
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5


def listed():
    return [
        # one token in front of the built-in perceptron's hidden width: latency
        dict(name="norm_one_row", op="norm", rows=1, n=1024, type="bf16", params="bf16", bias=True, train=False, autograd=False),
        # a minibatch of the policy study at its width, with gradients, as a captured step calls it: latency
        dict(name="norm_policy", op="norm", rows=128, n=128, type="fp32", params="fp32", bias=True, train=True, autograd=False),
        # rows of odd length, no bias
        dict(name="norm_odd", op="norm", rows=5003, n=1021, type="fp16", params="fp32", bias=False, train=True, autograd=False),
        # a large block's normalisation of 16 384 tokens, fp32 weights beside bf16 activations, through autograd
        dict(name="norm_block", op="norm", rows=16_384, n=8192, type="bf16", params="fp32", bias=True, train=True, autograd=True),
        # one token through a wide gated layer: the weights are the traffic
        dict(name="gated_one_row", op="gated", M=1, K=4096, N=8192, type="bf16", act="silu", bias=False, train=False, layout="nk", autograd=False),
        # a minibatch of 64 through the perceptron's sizes, weights stored in x out, with gradients
        dict(name="gated_perceptron", op="gated", M=64, K=784, N=1024, type="bf16", act="gelu", bias=True, train=True, layout="kn", autograd=False),
        # odd everywhere: no row of an operand but the first begins at a whole piece
        dict(name="gated_odd", op="gated", M=2003, K=1021, N=2731, type="fp16", act="relu", bias=True, train=True, layout="nk", autograd=False),
        # the first half of a large block on 8192 tokens, forward and backward
        dict(name="gated_block", op="gated", M=8192, K=2048, N=8192, type="bf16", act="silu", bias=False, train=True, layout="nk", autograd=True),
        # a small vocabulary and eight entries a row: latency
        dict(name="distill_small", op="distill", rows=64, vocab=1000, pad=0, k=8, type="fp32", teacher="fp32", masked=0.0, temperature=1.0, hard=0.0),
        # a few positions over a very large vocabulary: few rows, all of the chip
        dict(name="distill_few", op="distill", rows=8, vocab=131_072, pad=0, k=256, type="bf16", teacher="bf16", masked=0.0, temperature=2.0, hard=0.0),
        # odd vocabulary, labels beside the teacher at another temperature: two softmaxes of every row
        dict(name="distill_odd", op="distill", rows=2001, vocab=50_001, pad=0, k=50, type="fp16", teacher="fp16", masked=0.1, temperature=1.5, hard=0.3),
        # a micro-batch over a large vocabulary, prompts not counted
        dict(name="distill_large", op="distill", rows=4096, vocab=65_536, pad=0, k=64, type="bf16", teacher="bf16", masked=0.2, temperature=2.0, hard=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    op = rng.choice(["norm", "gated", "distill"])
    kind = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "norm":
        n = _log_int(rng, 1, 32_768)
        if rng.random() < 0.5:
            n = (n + 7) // 8 * 8
        rows = _log_int(rng, 1, min(100_000, 67_000_000 // n))
        return dict(op="norm", rows=rows, n=n, type=kind, params=rng.choice([kind, "fp32"]), bias=rng.random() < 0.7, train=rng.random() < 0.6,
                    autograd=rng.random() < 0.3)
    if op == "gated":
        M, K, N = (_log_int(rng, 1, 8192) for _ in range(3))
        if rng.random() < 0.5:
            K, N = (K + 7) // 8 * 8, (N + 7) // 8 * 8
        M = max(1, min(M, 8192 * 2048 * 8192 // (K * N)))
        return dict(op="gated", M=M, K=K, N=N, type=rng.choice(["bf16", "bf16", "fp16"]), act=rng.choice(["relu", "gelu", "silu"]), bias=rng.random() < 0.5,
                    train=rng.random() < 0.5, layout=rng.choice(["nk", "kn"]), autograd=rng.random() < 0.3)
    V = _log_int(rng, 10, 131_072)
    rows = _log_int(rng, 1, min(16_384, 100_000_000 // V))
    return dict(op="distill", rows=rows, vocab=V, pad=rng.choice([0, 0, 7, 64]), k=_log_int(rng, 1, min(256, max(1, V // 2))), type=kind,
                teacher=rng.choice([kind, "fp32"]), masked=rng.choice([0.0, 0.1, 0.4]), temperature=rng.choice([1.0, 1.5, 2.0, 4.0]),
                hard=rng.choice([0.0, 0.0, 0.1, 0.5]))


# ---- what the program holds before the call ---------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _norm_inputs(case, seed):
    g = _generator(seed)
    T, W, R, n = TYPES[case["type"]], TYPES[case["params"]], case["rows"], case["n"]
    # a residual stream: a scale and a small mean for each token, and some columns far from the others in all of them
    column = 0.5 * _normal(g, n) * (1.0 + 9.0 * (torch.rand(n, generator=g, device=DEVICE) < 0.01))
    scale, mean = torch.exp(0.5 * _normal(g, R, 1)), 0.3 * _normal(g, R, 1)
    x = torch.empty(R, n, dtype=T, device=DEVICE)
    for a in range(0, R, 4096):
        x[a:a + 4096] = (scale[a:a + 4096] * (_normal(g, min(4096, R - a), n) + column + mean[a:a + 4096])).to(T)
    w = (1.0 + 0.2 * _normal(g, n)).to(W)
    b = (0.1 * _normal(g, n)).to(W) if case["bias"] else None
    dy = None
    if case["train"]:
        dy = torch.empty(R, n, dtype=T, device=DEVICE)
        for a in range(0, R, 4096):
            dy[a:a + 4096] = _normal(g, min(4096, R - a), n).to(T)
    return dict(x=x, w=w, b=b, dy=dy)


def _gated_inputs(case, seed):
    g = _generator(seed)
    T, M, K, N = TYPES[case["type"]], case["M"], case["K"], case["N"]
    x = _normal(g, M, K).to(T)
    w = (1.5 * _normal(g, 2 * N, K) / math.sqrt(K)).to(T)
    if case["layout"] == "kn":                                # stored in x 2 out, seen as 2 out x in
        w = w.t().contiguous().t()
    b = (0.5 * _normal(g, 2 * N)).to(T) if case["bias"] else None
    dy = _normal(g, M, N).to(T) if case["train"] else None
    return dict(x=x, w=w, b=b, dy=dy)


def _distill_inputs(case, seed):
    g = _generator(seed)
    T, V, R, k = TYPES[case["type"]], case["vocab"], case["rows"], case["k"]
    end = V - V // 100 if V > 500 else V                      # the unused end of a padded vocabulary
    store = torch.zeros(R, V + case["pad"], dtype=T, device=DEVICE)
    tokens = torch.randint(0, end, (R,), generator=g, device=DEVICE)
    teacher_tokens = torch.empty(R, k, dtype=torch.int64, device=DEVICE)
    teacher_logits = torch.empty(R, k, dtype=TYPES[case["teacher"]], device=DEVICE)
    for a in range(0, R, 1024):
        z = 2.0 * _normal(g, min(1024, R - a), V)
        z.scatter_add_(1, tokens[a:a + 1024, None], 6.0 + 2.0 * _normal(g, len(z), 1))
        store[a:a + 1024, :V] = z.to(T)
        top = torch.topk(z[:, :end] + 0.7 * _normal(g, len(z), end), k, 1)
        teacher_tokens[a:a + 1024], teacher_logits[a:a + 1024] = top.indices, top.values.to(teacher_logits.dtype)
    store[:, end:V] = -math.inf
    # gradients in fp16 are scaled, as a mean over many rows would leave nothing of them
    scale = 64.0 * 2.0 ** int(math.log2(R)) if case["type"] == "fp16" else 1.0
    # a teacher that kept a share of its mass has fewer entries in some rows: the rest of them is not used
    used = torch.randint((k + 1) // 2, k + 1, (R, 1), generator=g, device=DEVICE)
    used = torch.where(torch.rand(R, 1, generator=g, device=DEVICE) < 0.5, used, k)
    teacher_tokens = torch.where(torch.arange(k, device=DEVICE) < used, teacher_tokens, -1)
    tokens = torch.where(torch.rand(R, generator=g, device=DEVICE) < case["masked"], -1, tokens)
    return dict(logits=store[:, :V], tokens=tokens, teacher_tokens=teacher_tokens, teacher_logits=teacher_logits, scale=scale)


def prepare(case, seed):
    s = {"norm": _norm_inputs, "gated": _gated_inputs, "distill": _distill_inputs}[case["op"]](case, seed)
    if case["op"] != "distill" and case["train"] and case["autograd"]:
        for k in ("x", "w", "b"):
            if s[k] is not None:
                s[k].requires_grad_()
    return dict(s, case=case)


# ---- one call ---------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    with torch.no_grad():
        return {"norm": _norm, "gated": _gated, "distill": _distill}[state["case"]["op"]](state)


def _run_own(s):
    import paper_1710_06952_amd as P
    c = s["case"]
    if c["op"] == "distill":
        r = P.distillation_loss_and_gradient(s["logits"], s["tokens"], s["teacher_tokens"], s["teacher_logits"], temperature=c["temperature"],
                                             hard_weight=c["hard"], loss_scale=s["scale"])
        return dict(loss=r.loss, dlogits=r.dlogits, divergences=r.divergences, log_probs=r.log_probs)
    need = (True, True, s["b"] is not None)
    if c["op"] == "norm":
        if not c["train"]:
            return dict(y=P.layer_norm(s["x"], s["w"], s["b"], eps=EPS))
        if c["autograd"]:
            y = P.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
        else:
            y, stats = P.layer_norm_forward(s["x"], s["w"], s["b"], eps=EPS)
            grads = P.layer_norm_gradients(s["dy"], s["x"], s["w"], stats, need=need)
    else:
        if not c["train"]:
            return dict(y=P.gated(s["x"], s["w"], s["b"], activation=c["act"]))
        if c["autograd"]:
            y = P.gated(s["x"], s["w"], s["b"], activation=c["act"])
        else:
            y, slopes = P.gated_forward(s["x"], s["w"], s["b"], activation=c["act"])
            grads = P.gated_gradients(s["dy"], s["x"], s["w"], slopes, need=need)
    if c["autograd"]:
        grads = torch.autograd.grad(y, [s[k] for k in ("x", "w", "b") if s[k] is not None], s["dy"])
    out = dict(y=y, dx=grads[0], dw=grads[1])
    if s["b"] is not None:
        out["db"] = grads[2]
    return out


# ---- the plain forms --------------------------------------------------------------------------------------------

def _norm(s):
    x, w = s["x"].float(), s["w"].float()
    T, W = s["x"].dtype, s["w"].dtype
    n = x.shape[1]
    x = x - x.sum(1, keepdim=True) / n
    r = 1.0 / torch.sqrt((x * x).sum(1, keepdim=True) / n + EPS)
    xh = x * r
    y = xh * w
    if s["b"] is not None:
        y = y + s["b"].float()
    out = dict(y=y.to(T))
    if s["case"]["train"]:
        dy = s["dy"].float()
        g = dy * w
        out["dx"] = (r * (g - g.sum(1, keepdim=True) / n - xh * ((g * xh).sum(1, keepdim=True) / n))).to(T)
        out["dw"] = (dy * xh).sum(0, dtype=torch.float64).to(W)
        if s["b"] is not None:
            out["db"] = dy.sum(0, dtype=torch.float64).to(W)
    return out


def _activation(z, act):
    """act(z) and its derivative."""
    if act == "relu":
        return z * (z > 0), (z > 0).to(z.dtype)
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return z * sig, sig * (1.0 + z * (1.0 - sig))


def _gated(s):
    x, w = s["x"].float(), s["w"].float()
    T, N = s["x"].dtype, s["case"]["N"]
    z = x @ w.t()
    if s["b"] is not None:
        z = z + s["b"].float()
    gate, slope = _activation(z[:, :N], s["case"]["act"])
    up = z[:, N:]
    out = dict(y=(gate * up).to(T))
    if s["case"]["train"]:
        dh = s["dy"].float()
        dz = torch.cat([dh * up * slope, dh * gate], 1)
        out |= dict(dx=(dz @ w).to(T), dw=(dz.t() @ x).to(T))
        if s["b"] is not None:
            out["db"] = dz.sum(0, dtype=torch.float64).to(T)
    return out


def _distill(s):
    c, tokens, entries = s["case"], s["tokens"], s["teacher_tokens"]
    T, a = c["temperature"], c["hard"]
    z = s["logits"].float()
    counted = tokens >= 0
    share = 1.0 / counted.sum().clamp(min=1).double()
    slope = share * s["scale"]
    top = z.amax(1, keepdim=True)
    e = torch.exp((z - top) * (1.0 / T))
    total = e.sum(1, keepdim=True)
    used = entries >= 0
    t = torch.where(used, s["teacher_logits"].double() * (1.0 / T), -math.inf)
    t = t - t.amax(1, keepdim=True)
    p = torch.exp(t)
    mass = p.sum(1, keepdim=True)
    p = p / mass
    at = entries.clamp(min=0)
    log_q = (z.gather(1, at) - top).double() * (1.0 / T) - torch.log(total.double())
    kl = torch.where(p > 0, p * (t - torch.log(mass) - log_q), 0.0).sum(1)
    soft = torch.where(counted, slope * (1.0 - a) * T, 0.0)[:, None]
    d = e * (soft / total).float()
    d.scatter_add_(1, at, (-soft * p).float())
    loss = (1.0 - a) * T * T * kl
    out = dict(divergences=torch.where(counted, kl, 0.0).float(), log_probs=None)
    if a > 0.0:
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        hot = tokens.clamp(min=0)[:, None]
        logp = ((z.gather(1, hot) - top).double() - torch.log(total.double()))[:, 0]
        hard = torch.where(counted, slope * a, 0.0)[:, None]
        d += e * (hard / total).float()
        d.scatter_add_(1, hot, -hard.float())
        loss = loss - a * logp
        out["log_probs"] = torch.where(counted, logp, 0.0).float()
    return dict(out, loss=(torch.where(counted, loss, 0.0).sum() * share).float(), dlogits=d.to(s["logits"].dtype))


# ---- the work and the same in 64 bits ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "norm":
        each, n = case["rows"] * case["n"], case["n"] * SIZE[case["params"]] * (2 if case["bias"] else 1)
        return dict(bytes=float(each * SIZE[case["type"]] * (4 if case["train"] else 2) + n * (2 if case["train"] else 1)),
                    flops=each * (20.0 if case["train"] else 8.0))
    if case["op"] == "gated":
        M, K, N = case["M"], case["K"], case["N"]
        n = M * K + 2 * N * K + M * N + (2 * N if case["bias"] else 0)
        if case["train"]:                                      # dh; dx, dw, db
            n += M * N + M * K + 2 * N * K + (2 * N if case["bias"] else 0)
        return dict(bytes=float(n * SIZE[case["type"]]), flops=4.0 * M * K * N * (3 if case["train"] else 1))
    two = case["hard"] > 0.0 and case["temperature"] != 1.0
    each = case["rows"] * case["vocab"]
    return dict(bytes=float(each * SIZE[case["type"]] * 2 + case["rows"] * case["k"] * (8 + SIZE[case["teacher"]])), flops=each * (10.0 if two else 6.0))


def exact(case, seed):
    return {"norm": _exact_norm, "gated": _exact_gated, "distill": _exact_distill}[case["op"]](case, seed)


def _exact_norm(case, seed):
    s = _norm_inputs(case, seed)
    R, n = case["rows"], case["n"]
    w, b = s["w"].double(), s["b"].double() if case["bias"] else None
    new = lambda: torch.empty(R, n, dtype=torch.float64, device=DEVICE)  # noqa: E731
    out = dict(y=new())
    if case["train"]:
        out |= dict(dx=new(), dw=torch.zeros_like(w))
        if case["bias"]:
            out["db"] = torch.zeros_like(w)
    for a in range(0, R, 4096):
        x = s["x"][a:a + 4096].double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        std = torch.sqrt(var + EPS)
        xh = (x - mean) / std
        out["y"][a:a + 4096] = xh * w + b if case["bias"] else xh * w
        if case["train"]:
            dy = s["dy"][a:a + 4096].double()
            g = dy * w
            out["dx"][a:a + 4096] = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) / std
            out["dw"] += (dy * xh).sum(0)
            if case["bias"]:
                out["db"] += dy.sum(0)
    return out


def _exact_gated(case, seed):
    s = {k: None if t is None else t.double() for k, t in _gated_inputs(case, seed).items()}
    N, act = case["N"], case["act"]
    z = torch.mm(s["x"], s["w"].t().contiguous())
    if case["bias"]:
        z += s["b"]
    g, u = z[:, :N], z[:, N:]
    if act == "relu":
        v, slope = g.clamp(min=0.0), torch.sign(g).clamp(min=0.0)
    elif act == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        v, slope = g * cdf, cdf + g * torch.exp(-g.square() / 2.0) / math.sqrt(2.0 * math.pi)
    else:
        sig = torch.sigmoid(g)
        v, slope = g * sig, sig + g * sig * (1.0 - sig)
    out = dict(y=v * u)
    if case["train"]:
        dz = torch.empty_like(z)
        dz[:, :N] = s["dy"] * u * slope
        dz[:, N:] = s["dy"] * v
        out |= dict(dx=torch.mm(dz, s["w"].contiguous()), dw=torch.mm(dz.t().contiguous(), s["x"]))
        if case["bias"]:
            out["db"] = dz.sum(0)
    return out


def _exact_distill(case, seed):
    s = _distill_inputs(case, seed)
    R, V, T, a = case["rows"], case["vocab"], case["temperature"], case["hard"]
    rows = torch.nonzero(s["tokens"] >= 0)[:, 0]
    n = max(1, len(rows))
    d = torch.zeros(R, V, dtype=torch.float64, device=DEVICE)
    kl, logp = torch.zeros(R, dtype=torch.float64, device=DEVICE), torch.zeros(R, dtype=torch.float64, device=DEVICE)
    for part in rows.split(1024):
        z = s["logits"][part].double()
        log_q = torch.log_softmax(z / T, 1)
        entries = s["teacher_tokens"][part]
        used = entries >= 0
        log_p = torch.log_softmax((s["teacher_logits"][part].double() / T).masked_fill(~used, -math.inf), 1)
        p = torch.zeros_like(z)
        where = used.nonzero()
        p.index_put_((where[:, 0], entries[used]), log_p[used].exp(), accumulate=True)
        kl[part] = (log_p.exp() * torch.where(used, log_p - log_q.gather(1, entries.clamp(min=0)), 0.0)).sum(1)
        d[part] = s["scale"] * (1.0 - a) * T / n * (log_q.exp() - p)
        if a > 0.0:
            log_q = torch.log_softmax(z, 1)
            hot = s["tokens"][part][:, None]
            logp[part] = log_q.gather(1, hot)[:, 0]
            d[part] += s["scale"] * a / n * log_q.exp().scatter_add(1, hot, torch.full_like(hot, -1, dtype=torch.float64))
    loss = ((1.0 - a) * T * T * kl.sum() - a * logp.sum()) / n
    return dict(divergences=kl, log_probs=logp if a > 0.0 else None, loss=loss, dlogits=d)
