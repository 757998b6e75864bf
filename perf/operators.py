"""The operators of a worker's own training step, as cases that can be timed and compared: dense layers, the
log-probabilities and losses over a vocabulary, and AdamW over many tensors at once.

A case names an operator and its sizes; ``prepare`` makes what a program holds before the call, ``run`` is one call:
through the framework's entry points where ``own`` is true, and else in plain torch operations in 32 bits (64 where
sums are long or a value stands next to a rounding border).  ``exact`` is the same result from the operator's
definition in 64 bits.

ops   dense       y = act(x w^T + b) + r, and with train its gradients for a given dy
      score       log-probability of one token a row
      policy      clipped policy loss with a KL term, and its gradient for the logits
      preference  paired log ratios of sequences of ragged lengths, and the gradient for the logits
      adamw       one AdamW step over all tensors of a model, states in 32 or 8 bits, clipped by the global norm
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # the built-in perceptron's four tensors, views of one flat fp32 vector as the engine keeps them: the smallest step
        dict(name="adamw_perceptron", op="adamw", tensors=4, total=814090, packed=True, param="fp32", grad="fp32", bits=32, masters=False,
             direction=False, clip=True),
        # the headline workload's 25.6 M parameters as the 161 tensors of a real network, fp32 throughout
        dict(name="adamw_32bit", op="adamw", tensors=161, total=25_600_000, packed=False, param="fp32", grad="fp32", bits=32, masters=False,
             direction=False, clip=True),
        # mixed precision with small states: bf16 parameters and gradients, fp32 masters, both moments in 8 bits
        dict(name="adamw_8bit", op="adamw", tensors=300, total=67_108_864, packed=False, param="bf16", grad="bf16", bits=8, masters=True,
             direction=False, clip=True),
        # reinforcement on a small vocabulary: latency
        dict(name="policy_small", op="policy", rows=64, vocab=1000, pad=0, type="fp32", masked=0.0, clip_low=0.2, clip_high=0.2, kl=0.05),
        # a micro-batch of sampled answers over a large vocabulary, prompts not counted
        dict(name="policy_large", op="policy", rows=4096, vocab=65_536, pad=0, type="bf16", masked=0.2, clip_low=0.2, clip_high=0.28, kl=0.02),
        # four short pairs, fp32 logits
        dict(name="preference_small", op="preference", pairs=4, longest=24, vocab=2048, pad=0, type="fp32", masked=0.1, beta=0.1, smoothing=0.0),
        # ragged pairs over a vocabulary of odd size: rows begin anywhere
        dict(name="preference_large", op="preference", pairs=8, longest=512, vocab=50_001, pad=0, type="bf16", masked=0.3, beta=0.1, smoothing=0.05),
        # the next token of a few sequences over a very large vocabulary: few rows, all of the chip
        dict(name="score_few", op="score", rows=8, vocab=131_072, pad=0, type="bf16", masked=0.0),
        # log-probabilities of a batch under the frozen model, padded rows
        dict(name="score_many", op="score", rows=8000, vocab=32_000, pad=64, type="fp16", masked=0.1),
        # one token through a wide layer: the weights are the traffic
        dict(name="dense_one_row", op="dense", M=1, K=4096, N=8192, type="bf16", act="silu", bias=True, residual=False, train=False, layout="nk"),
        # the perceptron's first layer on one minibatch, weights stored in x hidden as the engine stores them, with gradients
        dict(name="dense_perceptron", op="dense", M=64, K=784, N=1024, type="bf16", act="relu", bias=True, residual=False, train=True, layout="kn"),
        # a feed-forward layer of a large block on 8192 tokens with its residual stream, forward and backward
        dict(name="dense_block", op="dense", M=8192, K=2048, N=8192, type="bf16", act="gelu", bias=True, residual=True, train=True, layout="nk"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    op = rng.choice(["dense", "dense", "score", "policy", "preference", "adamw", "adamw"])
    kind = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    masked = rng.choice([0.0, 0.1, 0.4])
    if op == "dense":
        M, K, N = (_log_int(rng, 1, 8192) for _ in range(3))
        if rng.random() < 0.5:
            K, N = (K + 7) // 8 * 8, (N + 7) // 8 * 8
        return dict(op="dense", M=M, K=K, N=N, type=rng.choice(["bf16", "fp16"]), act=rng.choice(["none", "relu", "gelu", "silu"]),
                    bias=rng.random() < 0.7, residual=rng.random() < 0.5, train=rng.random() < 0.5, layout=rng.choice(["nk", "kn"]))
    if op == "adamw":
        total = _log_int(rng, 1000, 40_000_000)
        param = rng.choice(["fp32", "bf16", "fp16"])
        return dict(op="adamw", tensors=min(_log_int(rng, 1, 400), total // 10), total=total, packed=rng.random() < 0.5, param=param,
                    grad=rng.choice(["fp32", param]), bits=rng.choice([32, 8]), masters=param != "fp32" and rng.random() < 0.7,
                    direction=rng.random() < 0.3, clip=rng.random() < 0.7)
    V = _log_int(rng, 10, 131_072)
    rows = _log_int(rng, 1, min(16_384, 100_000_000 // V))
    pad = rng.choice([0, 0, 7, 64])
    if op == "score":
        return dict(op="score", rows=rows, vocab=V, pad=pad, type=kind, masked=masked)
    if op == "policy":
        return dict(op="policy", rows=rows, vocab=V, pad=pad, type=kind, masked=masked, clip_low=0.2, clip_high=rng.choice([0.2, 0.3]),
                    kl=rng.choice([0.0, 0.05, 0.5]))
    pairs = _log_int(rng, 1, max(2, min(64, rows // 4)))
    return dict(op="preference", pairs=pairs, longest=max(1, rows // (2 * pairs)), vocab=V, pad=pad, type=kind, masked=masked,
                beta=rng.choice([0.05, 0.1, 0.3]), smoothing=rng.choice([0.0, 0.1]))


# ---- what the program holds before the call ---------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


BETAS, EPS, LR, STEPS_BEFORE, GRAD_SCALE = (0.9, 0.999), 1e-8, 1e-3, 41, 0.5


def _sizes(case):
    """Sizes of the tensors of a model: few large, many small; the built-in perceptron's own where they fit."""
    if case["tensors"] == 4 and case["total"] == 784 * 1024 + 1024 + 1024 * 10 + 10:
        return [784 * 1024, 1024, 1024 * 10, 10]
    rng = random.Random(case["total"] * 1009 + case["tensors"])
    share = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["tensors"])]
    sizes = [max(1, int(case["total"] * s / sum(share))) for s in share]
    sizes[sizes.index(max(sizes))] += case["total"] - sum(sizes)
    return sizes


def _spread(flat, sizes, starts, length):
    """A vector of tensors one behind the other, each moved to its own start."""
    out = torch.zeros(length, dtype=flat.dtype, device=flat.device)
    at = 0
    for n, s in zip(sizes, starts):
        out[s:s + n] = flat[at:at + n]
        at += n
    return out


def _codes_on_device():
    """The values that e4m3 holds, not negative, ascending."""
    return torch.arange(127, dtype=torch.uint8, device=DEVICE).view(torch.float8_e4m3fn).to(torch.float64)


def _block_exponent(x):
    """floor(log2) of the largest magnitude of each block of 256, not under -43, less 7: the exponent of its scale."""
    return (torch.frexp(x.abs().view(-1, 256).amax(1))[1] - 1).clamp(min=-43) - 7


def _adamw_inputs(case, seed):
    g = _generator(seed)
    sizes = _sizes(case)
    state_starts, n = [], 0
    for s in sizes:
        state_starts.append(n)
        n += -(-s // 256) * 256
    total = sum(sizes)
    starts = [sum(sizes[:i]) for i in range(len(sizes))] if case["packed"] else state_starts
    length = total if case["packed"] else n
    spread = lambda x, to, size: _spread(x, sizes, to, size)  # noqa: E731
    scale = torch.exp(_normal(g, total))                      # gradients of different magnitude from one element to the next
    grad = 0.01 * scale * _normal(g, total)
    m = 0.003 * scale * _normal(g, total)
    v = (0.01 * scale) ** 2 * (0.5 + torch.rand(total, generator=g, device=DEVICE))
    p = 0.05 * _normal(g, total)
    m, v = spread(m, state_starts, n), spread(v, state_starts, n)
    if case["bits"] == 8:                                     # moments that the 8-bit form holds
        codes = _codes_on_device()
        km, kv = _block_exponent(m.double()), _block_exponent(v.double().sqrt())
        ym, yv = torch.ldexp(m.double().view(-1, 256), -km[:, None]), torch.ldexp(v.double().sqrt().view(-1, 256), -kv[:, None])
        m = (torch.ldexp(codes[torch.bucketize(ym.abs(), (codes[1:] + codes[:-1]) / 2)] * ym.sign(), km[:, None])).reshape(-1).float()
        r = torch.where(yv > 0, codes[torch.bucketize(yv, (codes[1:] + codes[:-1]) / 2).clamp(min=1)], 0.0)
        v = torch.ldexp(r, kv[:, None]).reshape(-1).square().float()
    P, G = TYPES[case["param"]], TYPES[case["grad"]]
    master = spread(p, starts, length) if case["masters"] else None
    return dict(sizes=sizes, starts=starts, state_starts=state_starts, state_length=n, length=length, decay=[0.0 if s < 5000 else 0.1 for s in sizes],
                p=spread(p.to(P), starts, length), g=spread(grad.to(G), starts, length), master=master, m=m, v=v,
                out=torch.zeros(length, device=DEVICE) if case["direction"] else None,
                max_norm=0.5 * GRAD_SCALE * float(grad.norm()) if case["clip"] else 0.0, seed=int(seed) * 2654435761 + 12345)


def _loss_inputs(case, seed):
    g = _generator(seed)
    T, V = TYPES[case["type"]], case["vocab"]
    if case["op"] == "preference":
        longest = case["longest"]
        lengths = [random.Random(longest * 31 + case["pairs"] + 7 * q).randint(1, longest) for q in range(2 * case["pairs"])]
        if len(lengths) > 4:
            lengths[3] = 0                                    # an empty answer
        offsets = torch.tensor([sum(lengths[:q]) for q in range(len(lengths) + 1)], device=DEVICE)
        R = sum(lengths)
    else:
        R, offsets = case["rows"], None
    store = torch.zeros(R, V + case["pad"], dtype=T, device=DEVICE)
    tokens = torch.randint(0, V, (R,), generator=g, device=DEVICE)
    boost = 6.0 + 2.0 * _normal(g, R)
    for a in range(0, R, 1024):
        z = 2.0 * _normal(g, min(1024, R - a), V)
        z.scatter_add_(1, tokens[a:a + 1024, None], boost[a:a + 1024, None])
        store[a:a + 1024, :V] = z.to(T)
    logits = store[:, :V]
    if V > 500:                                               # the unused end of a padded vocabulary
        store[:, V - V // 100:V] = -math.inf
        tokens = tokens.clamp(max=V - V // 100 - 1)
    tokens = torch.where(torch.rand(R, generator=g, device=DEVICE) < case["masked"], -1, tokens)
    state = dict(logits=logits, tokens=tokens, offsets=offsets)
    if case["op"] == "score":
        return state
    logp = torch.empty(R, device=DEVICE)
    for a in range(0, R, 1024):
        z = logits[a:a + 1024].float()
        logp[a:a + 1024] = z.gather(1, tokens[a:a + 1024, None].clamp(min=0))[:, 0] - torch.logsumexp(z, 1)
    logp = torch.where(tokens >= 0, logp, 0.0)
    if case["op"] == "policy":
        state |= dict(old=logp + 0.2 * _normal(g, R), ref=logp + 0.5 * _normal(g, R) if case["kl"] else None,
                      advantages=0.25 + _normal(g, R))
    else:
        sums = torch.stack([x.sum() for x in logp.double().split(lengths)])
        state |= dict(ref=(sums + 3.0 * _normal(g, len(lengths))).float())
    return state


def _dense_inputs(case, seed):
    g = _generator(seed)
    T, M, K, N = TYPES[case["type"]], case["M"], case["K"], case["N"]
    x = _normal(g, M, K).to(T)
    w = (_normal(g, N, K) / math.sqrt(K)).to(T)
    if case["layout"] == "kn":                                # stored in x out, seen as out x in
        w = w.t().contiguous().t()
    b = (0.5 * _normal(g, N)).to(T) if case["bias"] else None
    r = _normal(g, M, N).to(T) if case["residual"] else None
    dy = _normal(g, M, N).to(T) if case["train"] else None
    return dict(x=x, w=w, b=b, r=r, dy=dy)


def prepare(case, seed):
    if case["op"] == "adamw":
        s = _adamw_inputs(case, seed)
        place = torch.zeros(s["length"], dtype=torch.int64, device=DEVICE)   # of each stored element in the state
        decay = torch.zeros(s["state_length"], device=DEVICE)
        for n, a, b, wd in zip(s["sizes"], s["starts"], s["state_starts"], s["decay"]):
            place[a:a + n] = torch.arange(b, b + n, device=DEVICE)
            decay[b:b + n] = wd
        s |= dict(place=place if case["packed"] else None, decay_of=decay, steps=STEPS_BEFORE)
        if own:
            import paper_1710_06952_amd as P
            views = lambda x: None if x is None else [x[a:a + n] for a, n in zip(s["starts"], s["sizes"])]  # noqa: E731
            s["optimizer"] = P.AdamW(views(s["p"]), views(s["g"]), lr=LR, betas=BETAS, eps=EPS, weight_decay=s["decay"], state_bits=case["bits"],
                                     masters=views(s["master"]), out=views(s["out"]), seed=s["seed"])
            s["optimizer"].load_moments(s["m"], s["v"], STEPS_BEFORE)
    elif case["op"] == "dense":
        s = _dense_inputs(case, seed)
        if case["train"]:
            for k in ("x", "w", "b", "r"):
                if s[k] is not None:
                    s[k].requires_grad_()
    else:
        s = _loss_inputs(case, seed)
    return dict(s, case=case)


# ---- one call ---------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    with torch.no_grad():
        return {"adamw": _adamw, "dense": _dense, "score": _score, "policy": _policy, "preference": _preference}[state["case"]["op"]](state)


def _run_own(s):
    import paper_1710_06952_amd as P
    c = s["case"]
    if c["op"] == "adamw":
        norm = s["optimizer"].step(max_norm=s["max_norm"], grad_scale=GRAD_SCALE)
        m, v = s["optimizer"].moments()
        return dict(p=s["p"], master=s["master"], out=s["out"], m=m, v=v, norm=norm)
    if c["op"] == "dense":
        y = P.dense(s["x"], s["w"], s["b"], residual=s["r"], activation=c["act"])
        if not c["train"]:
            return dict(y=y)
        names = [k for k in ("x", "w", "b", "r") if s[k] is not None]
        grads = torch.autograd.grad(y, [s[k] for k in names], s["dy"])
        return dict({"d" + k: d for k, d in zip(names, grads)}, y=y)
    if c["op"] == "score":
        return dict(log_probs=P.token_log_probs(s["logits"], s["tokens"]))
    if c["op"] == "policy":
        r = P.policy_loss_and_gradient(s["logits"], s["tokens"], s["old"], s["advantages"], s["ref"], clip=(c["clip_low"], c["clip_high"]), kl_coef=c["kl"])
        return dict(loss=r.loss, dlogits=r.dlogits, log_probs=r.log_probs)
    r = P.preference_loss_and_gradient(s["logits"], s["tokens"], s["offsets"], s["ref"], beta=c["beta"], label_smoothing=c["smoothing"])
    return dict(loss=r.loss, dlogits=r.dlogits, log_probs=r.log_probs, margins=r.margins)


# ---- the plain forms --------------------------------------------------------------------------------------------

def _activation(z, act):
    """act(z) and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z * (z > 0), (z > 0).to(z.dtype)
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-z))
    return z * sig, sig * (1.0 + z * (1.0 - sig))


def _dense(s):
    x, w = s["x"].float(), s["w"].float()
    T = s["x"].dtype
    z = x @ w.t()
    if s["b"] is not None:
        z = z + s["b"].float()
    y, slope = _activation(z, s["case"]["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    out = dict(y=y.to(T))
    if s["case"]["train"]:
        dz = s["dy"].float() * slope
        out |= dict(dx=(dz @ w).to(T), dw=(dz.t() @ x).to(T))
        if s["b"] is not None:
            out["db"] = dz.sum(0, dtype=torch.float64).to(T)
        if s["r"] is not None:
            out["dr"] = s["dy"]
    return out


def _log_probs(logits, tokens):
    """Of the tokens (0 where there is none), and exp(z - largest) with its sum."""
    z = logits.float()
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = z.gather(1, tokens.clamp(min=0)[:, None])
    logp = ((at - top).double() - torch.log(total.double()))[:, 0]
    return torch.where(tokens >= 0, logp, 0.0), e, total


def _logit_gradient(coef, e, total, tokens, T):
    d = e * (-coef[:, None] / total)
    d.scatter_add_(1, tokens.clamp(min=0)[:, None], coef[:, None])
    return d.to(T)


def _score(s):
    return dict(log_probs=_log_probs(s["logits"], s["tokens"])[0].float())


def _policy(s):
    c, tokens = s["case"], s["tokens"]
    logp, e, total = _log_probs(s["logits"], tokens)
    counted = tokens >= 0
    share = 1.0 / counted.sum().clamp(min=1).double()
    ratio = torch.exp(logp - s["old"])
    free = ratio * s["advantages"]
    held = ratio.clamp(1.0 - c["clip_low"], 1.0 + c["clip_high"]) * s["advantages"]
    loss, slope = -torch.minimum(free, held), torch.where(free <= held, -free, 0.0)
    if s["ref"] is not None:
        d = s["ref"] - logp
        loss = loss + c["kl"] * (torch.exp(d) - d - 1.0)
        slope = slope + c["kl"] * (1.0 - torch.exp(d))
    loss = (torch.where(counted, loss, 0.0).sum() * share).float()
    coef = (torch.where(counted, slope, 0.0) * share).float()
    return dict(loss=loss, dlogits=_logit_gradient(coef, e, total, tokens, s["logits"].dtype), log_probs=logp.float())


def _preference(s):
    c, tokens, offsets = s["case"], s["tokens"], s["offsets"]
    logp, e, total = _log_probs(s["logits"], tokens)
    before = torch.nn.functional.pad(logp.cumsum(0), (1, 0))
    sums = before[offsets[1:]] - before[offsets[:-1]]
    pairs = c["pairs"]
    ratio = sums - s["ref"]
    margin = c["beta"] * (ratio[:pairs] - ratio[pairs:])
    low = lambda x: torch.log1p(torch.exp(-x.abs())) - x.clamp(max=0.0)  # noqa: E731  -log sigma(x)
    eps = c["smoothing"]
    loss = ((1.0 - eps) * low(margin) + eps * low(-margin)).mean().float()
    slope = c["beta"] / pairs * (eps - 1.0 / (1.0 + torch.exp(margin)))     # of the loss, for the chosen sequence's sum
    of = torch.bucketize(torch.arange(len(tokens), device=tokens.device), offsets[1:], right=True)
    coef = torch.where(tokens >= 0, torch.cat([slope, -slope])[of], 0.0).float()
    return dict(loss=loss, dlogits=_logit_gradient(coef, e, total, tokens, s["logits"].dtype), log_probs=sums.float(), margins=margin.float())


def _philox(length, step, seed):
    """The library's counter generator (Philox4x32-10, stream 3): one 32-bit word for each element of a state."""
    lane = torch.arange((length + 3) // 4, device=DEVICE)
    low = 0xFFFFFFFF
    c = [lane & low, lane >> 32, torch.full_like(lane, step & low), torch.full_like(lane, ((step >> 32) & 0xFFFFFF) | (3 << 24))]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(c, 1).reshape(-1)[:length]


def _eight_bits(x, up, root):
    """Values of blocks of 256 (64 bits) as e4m3 with the block's scale holds them, rounded up where the share of the way to the
    next code and `up` come to one.  root: the square root is held, rounded so that its square keeps its mean, and never to zero."""
    held = x.sqrt() if root else x.abs()
    k = _block_exponent(held)[:, None]
    y = torch.ldexp(held.view(-1, 256), -k)
    quantum = torch.ldexp(torch.ones_like(y), (torch.frexp(y)[1] - 1).clamp(min=-6) - 3)
    lo = torch.floor(y / quantum) * quantum
    hi = lo + quantum
    share = (torch.ldexp(x.view(-1, 256), -2 * k) - lo * lo) / (hi * hi - lo * lo) if root else (y - lo) / quantum
    q = torch.where(share + up.view(-1, 256) >= 1.0, hi, lo)
    if root:
        return torch.ldexp(torch.where(y > 0, q.clamp(min=2.0 ** -9), 0.0), k).square().reshape(-1).float()
    return (torch.ldexp(q, k).reshape(-1) * x.sign()).float()


def _adamw(s):
    c, place = s["case"], s["place"]
    gather = lambda x: x.float() if place is None else torch.zeros_like(s["m"]).index_copy_(0, place, x.float())  # noqa: E731
    back = lambda x: x if place is None else x[place]  # noqa: E731
    g = gather(s["g"]) * GRAD_SCALE
    norm = g.square().sum(dtype=torch.float64).sqrt()
    if c["clip"]:
        g = g * (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    s["steps"] += 1
    t, (b1, b2) = s["steps"], BETAS
    m, v = b1 * s["m"] + (1.0 - b1) * g, b2 * s["v"] + (1.0 - b2) * g * g
    u = (m / (1.0 - b1 ** t)) / ((v / (1.0 - b2 ** t)).sqrt() + EPS)
    if c["bits"] == 8:
        word = _philox(len(m), t, s["seed"])
        g, m, v = g.double(), s["m"].double(), s["v"].double()
        s["m"] = _eight_bits(b1 * m + (1.0 - b1) * g, ((word >> 16) + 0.5) / 65536.0, False)
        s["v"] = _eight_bits(b2 * v + (1.0 - b2) * g * g, ((word & 0xFFFF) + 0.5) / 65536.0, True)
    else:
        s["m"], s["v"] = m, v
    p = gather(s["p"] if s["master"] is None else s["master"])
    if c["direction"]:
        s["out"].copy_(back(u + s["decay_of"] * p))
    else:
        p = back(p - LR * (u + s["decay_of"] * p))
        s["p"].copy_(p)
        if s["master"] is not None:
            s["master"].copy_(p)
    held = (lambda x: x.to(torch.bfloat16)) if c["bits"] == 8 else lambda x: x      # what eight bits stand for is exact in bf16
    return dict(p=s["p"], master=s["master"], out=s["out"], m=held(s["m"]), v=held(s["v"]), norm=norm.float() if c["clip"] else None)


# ---- the work and the same in 64 bits ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "dense":
        M, K, N, b = case["M"], case["K"], case["N"], SIZE[case["type"]]
        n = M * K + N * K + M * N * (2 if case["residual"] else 1) + (N if case["bias"] else 0)
        if case["train"]:                                      # dy; dx, dw, db
            n += M * N + M * K + N * K + (N if case["bias"] else 0)
        return dict(bytes=float(n * b), flops=2.0 * M * K * N * (3 if case["train"] else 1))
    if case["op"] == "adamw":
        p, g, st = SIZE[case["param"]], SIZE[case["grad"]], case["bits"] / 8
        model = (4 if case["masters"] else p)
        n = g + 4 * st + model                                  # gradient; both moments read and written; the model read ...
        n += 4 if case["direction"] else model + (p if case["masters"] else 0)
        return dict(bytes=float(n * case["total"]), flops=15.0 * case["total"])
    rows = case["rows"] if case["op"] != "preference" else case["pairs"] * (case["longest"] + 1)
    n = rows * case["vocab"] * SIZE[case["type"]]
    return dict(bytes=float(n * (1 if case["op"] == "score" else 2)), flops=rows * case["vocab"] * (4.0 if case["op"] == "score" else 6.0))


def exact(case, seed):
    return {"dense": _exact_dense, "adamw": _exact_adamw, "score": _exact_loss, "policy": _exact_loss,
            "preference": _exact_loss}[case["op"]](case, seed)


def _exact_dense(case, seed):
    s = {k: None if t is None else t.double() for k, t in _dense_inputs(case, seed).items()}
    z = torch.mm(s["x"], s["w"].t().contiguous())
    if case["bias"]:
        z += s["b"]
    act = case["act"]
    if act == "none":
        y, slope = z, torch.ones_like(z)
    elif act == "relu":
        y, slope = z.clamp(min=0.0), torch.sign(z).clamp(min=0.0)
    elif act == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        y, slope = z * cdf, cdf + z * torch.exp(-z.square() / 2.0) / math.sqrt(2.0 * math.pi)
    else:
        sig = torch.sigmoid(z)
        y, slope = z * sig, sig + z * sig * (1.0 - sig)
    out = dict(y=y + s["r"] if case["residual"] else y)
    if case["train"]:
        dz = s["dy"] * slope
        out |= dict(dx=torch.mm(dz, s["w"].contiguous()), dw=torch.mm(dz.t().contiguous(), s["x"]))
        if case["bias"]:
            out["db"] = dz.sum(0)
        if case["residual"]:
            out["dr"] = s["dy"]
    return out


def _exact_loss(case, seed):
    s = _loss_inputs(case, seed)
    tokens, R = s["tokens"], len(s["tokens"])
    lse = torch.empty(R, dtype=torch.float64, device=DEVICE)
    for a in range(0, R, 1024):
        lse[a:a + 1024] = torch.logsumexp(s["logits"][a:a + 1024].double(), 1)
    hit = torch.nonzero(tokens >= 0)[:, 0]
    logp = torch.zeros(R, dtype=torch.float64, device=DEVICE)
    logp[hit] = s["logits"][hit, tokens[hit]].double() - lse[hit]
    if case["op"] == "score":
        return dict(log_probs=logp)
    slope = torch.zeros_like(logp)
    if case["op"] == "policy":
        l, A = logp[hit], s["advantages"][hit].double()
        rho = torch.exp(l - s["old"][hit].double())
        inside = torch.where(A >= 0, rho <= 1.0 + case["clip_high"], rho >= 1.0 - case["clip_low"])
        edge = torch.where(A >= 0, 1.0 + case["clip_high"], 1.0 - case["clip_low"])
        terms, d = -A * torch.where(inside, rho, edge), torch.where(inside, -A * rho, 0.0)
        if s["ref"] is not None:
            gap = s["ref"][hit].double() - l
            terms, d = terms + case["kl"] * (torch.expm1(gap) - gap), d - case["kl"] * torch.expm1(gap)
        n = max(1, len(hit))
        slope[hit] = d / n
        out = dict(loss=terms.sum() / n, log_probs=logp)
    else:
        ends = s["offsets"].tolist()
        pairs = case["pairs"]
        sums = torch.stack([logp[a:b].sum() for a, b in zip(ends[:-1], ends[1:])])
        over = sums - s["ref"].double()
        margin = case["beta"] * (over[:pairs] - over[pairs:])
        soft = torch.nn.functional.softplus
        loss = ((1.0 - case["smoothing"]) * soft(-margin) + case["smoothing"] * soft(margin)).sum() / pairs
        by = (torch.sigmoid(margin) - (1.0 - case["smoothing"])) * case["beta"] / pairs
        for q, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
            slope[a:b] = by[q] if q < pairs else -by[q - pairs]
        slope[tokens < 0] = 0.0
        out = dict(loss=loss, log_probs=sums, margins=margin)
    d = torch.empty(R, case["vocab"], dtype=torch.float64, device=DEVICE)
    for a in range(0, R, 1024):
        d[a:a + 1024] = -slope[a:a + 1024, None] * torch.exp(s["logits"][a:a + 1024].double() - lse[a:a + 1024, None])
    d[hit, tokens[hit]] += slope[hit]
    return dict(out, dlogits=d)


def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    parts = lambda x: [x[a:a + n].double() for a, n in zip(s["starts"], s["sizes"])]  # noqa: E731
    scale = torch.tensor(GRAD_SCALE, dtype=torch.float64, device=DEVICE)
    norm = scale * s["g"].double().norm()
    if case["clip"]:
        scale = scale * min(1.0, s["max_norm"] / (float(norm) + 1e-6))
    t = STEPS_BEFORE + 1
    c1, c2 = 1.0 - BETAS[0] ** t, 1.0 - BETAS[1] ** t
    old = s["p"] if s["master"] is None else s["master"]
    new = old.double()
    direction = torch.zeros_like(new) if case["direction"] else None
    M, V = s["m"].double(), s["v"].double()
    for g, p, a, b, wd in zip(parts(s["g"]), parts(old), s["starts"], s["state_starts"], s["decay"]):
        n = len(g)
        m, v = M[b:b + n], V[b:b + n]                           # views: updated in place
        m += (1.0 - BETAS[0]) * (scale * g - m)
        v += (1.0 - BETAS[1]) * ((scale * g) ** 2 - v)
        step = m / c1 / (torch.sqrt(v / c2) + EPS) + wd * p
        if case["direction"]:
            direction[a:a + n] = step
        else:
            new[a:a + n] = p - LR * step
    if case["bits"] == 8:                                       # the nearest codes on both sides, and the draw between them
        codes, word = _codes_on_device(), _philox(len(M), t, s["seed"])
        for x, u, power in ((M, word >> 16, 1), (V, word & 0xFFFF, 2)):
            size = x.abs() ** (1.0 / power)
            unit = torch.exp2(_block_exponent(size).double()).repeat_interleave(256)
            below = (torch.bucketize(size / unit, codes, right=True) - 1).clamp(0, 125)
            lo, hi = codes[below] * unit, codes[below + 1] * unit
            share = (x.abs() - lo ** power) / (hi ** power - lo ** power)
            code = torch.where(share + (u + 0.5) / 65536.0 >= 1.0, hi, lo)
            if power == 2:
                code = torch.where(x > 0, torch.maximum(code, codes[1] * unit), code)
            x.copy_(code ** power * x.sign())
    return dict(p=s["p"].double() if case["direction"] else new, master=None if s["master"] is None else old.double() if case["direction"] else new,
                out=direction, m=M, v=V, norm=norm if case["clip"] else None)
