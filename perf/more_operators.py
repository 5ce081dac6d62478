"""Operators around a trainer's step on distilled rollouts, measured: a teacher's top logits, distillation from them, and cross
entropy straight from hidden states and an lm-head's weights, at the sizes that a program around this library meets.

A case names an operator (`op`):

  top      top_logits: the k largest logits of every row, and its log-sum-exp
  distill  distill_top: loss and gradient of a student's logits against a teacher's top logits
  linear   linear_ce, linear_ce_bwd: the cross entropy of hidden states through an lm-head, without [N, V] logits; its gradients

`own` false: the plain forms, elementary torch operations.  `own` true: the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
LEAST_REST = 2.0 ** -20          # a teacher's rest is never taken for less


def listed():
    return [
        # a teacher's decoding step: the rows of a few sequences
        dict(name="top_8", op="top", N=8, V=151936, k=64, dtype="bf16", temperature=1.0),
        # a teacher's forward pass over a training batch
        dict(name="top_4096", op="top", N=4096, V=151936, k=64, dtype="bf16", temperature=1.0),
        # fp32 rows of an odd vocabulary, long lists, a temperature
        dict(name="top_f32", op="top", N=1500, V=32003, k=100, dtype="f32", temperature=1.25),
        # a small batch on the small vocabulary; the teacher's list taken as all there is
        dict(name="distill_16", op="distill", N=16, V=32000, k=16, dtype="bf16", reverse=False, rest=False, temperature=1.0),
        # a trainer's batch, forward divergence, the rest of the vocabulary as one event
        dict(name="distill_4096", op="distill", N=4096, V=151936, k=64, dtype="bf16", reverse=False, rest=True, temperature=1.0),
        # reverse divergence, the longest lists
        dict(name="distill_reverse", op="distill", N=2048, V=151936, k=128, dtype="bf16", reverse=True, rest=True, temperature=1.0),
        # fp32 rows of an odd vocabulary, ragged lists
        dict(name="distill_f32", op="distill", N=1000, V=32003, k=20, dtype="f32", reverse=False, rest=True, temperature=0.9),
        # a handful of positions: the weights' bytes count, not the products
        dict(name="linear_64", op="linear", N=64, d=1024, V=32000, masked=0, routed=False, backward=True, temperature=1.0),
        # the loss alone (evaluation of a batch)
        dict(name="linear_loss", op="linear", N=4096, d=2560, V=151936, masked=0, routed=False, backward=False, temperature=1.0),
        # a trainer's step from routing metadata, an eighth of the positions masked
        dict(name="linear_4096", op="linear", N=4096, d=2560, V=151936, masked=512, routed=True, backward=True, temperature=1.0),
        # odd numbers of positions, vocabulary entries and features; a temperature
        dict(name="linear_odd", op="linear", N=1531, d=1096, V=32003, masked=100, routed=False, backward=True, temperature=1.1),
        # the largest batch
        dict(name="linear_8192", op="linear", N=8192, d=2560, V=151936, masked=0, routed=False, backward=True, temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("top", "top", "distill", "distill", "distill", "linear", "linear"))
    temperature = rng.choice((1.0, 1.0, 0.75, 1.25))
    if op == "linear":
        d, V = 8 * _log_int(rng, 16, 512), _log_int(rng, 1000, 152000)
        N = _log_int(rng, 16, max(17, min(8192, int(6e12 / 2 / d / V))))
        return dict(op=op, N=N, d=d, V=V, masked=rng.choice((0, 0, rng.randint(0, N // 2))), routed=rng.random() < 0.5,
                    backward=rng.random() < 0.75, temperature=temperature)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    V = _log_int(rng, 1000, 152000)
    N = _log_int(rng, 1, max(2, min(8192, int((6e8 if dtype == "bf16" else 3e8) / V))))
    case = dict(op=op, N=N, V=V, k=_log_int(rng, 1, 128), dtype=dtype, temperature=temperature)
    if op == "distill":
        case["reverse"] = rng.random() < 0.4
        case["rest"] = case["reverse"] or rng.random() < 0.6
    return case


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * 11 + seed)


def _type(case):
    return F32 if case.get("dtype") == "f32" else BF16


def _logits(gen, N, V):
    """Gaussian logits with a bias by rank, in float32."""
    x = torch.rand((N, V), generator=gen, device=DEV).mul_(V).log1p_().mul_(-1.1)
    return x.add_(torch.randn((N, V), generator=gen, device=DEV), alpha=2.0)


def prepare(case, seed):
    gen, op, N, V = _gen(seed), case["op"], case["N"], case["V"]
    s = dict(case=case)
    if op == "linear":
        d = case["d"]
        s["weight"] = (2.0 / math.sqrt(d) * torch.randn((V, d), generator=gen, device=DEV)).to(BF16)
        s["target"] = torch.randint(0, V, (N,), generator=gen, device=DEV, dtype=torch.int32)
        # hidden states lean towards their targets, some more than others
        lean = 4.0 * torch.rand((N, 1), generator=gen, device=DEV)
        s["hidden"] = (torch.randn((N, d), generator=gen, device=DEV) + lean * s["weight"][s["target"].long()].float()).to(BF16)
        s["mask"] = None
        if case["masked"]:
            s["mask"] = (torch.randperm(N, generator=gen, device=DEV) >= case["masked"]).to(torch.uint8)
        s["corrected"] = s["teacher_top1"] = s["advantage"] = None
        if case["routed"]:
            s["corrected"] = (torch.rand(N, generator=gen, device=DEV) < 0.2).to(torch.uint8)
            s["teacher_top1"] = torch.randint(0, V, (N,), generator=gen, device=DEV, dtype=torch.int32)
            s["advantage"] = torch.randn(N, generator=gen, device=DEV)
        s["grad_scale"] = 1.0 / max(1, N - case["masked"])
        return s
    x = _logits(gen, N, V)
    s["logits"] = x.to(_type(case), copy=True)
    if op == "distill":
        k = case["k"]
        t = x.mul_(0.8).add_(torch.randn((N, V), generator=gen, device=DEV))      # the teacher's row, of which k entries are kept
        logit, token = torch.topk(t, k, dim=1)
        s["lse"] = torch.logsumexp(t / case["temperature"], 1) if case["rest"] else None
        # lists of different lengths: a quarter of the rows keep some of their entries
        keep = torch.where(torch.rand((N, 1), generator=gen, device=DEV) < 0.25, torch.rand((N, 1), generator=gen, device=DEV) * k, float(k))
        there = torch.arange(k, device=DEV) < keep
        s["token"] = torch.where(there, token, -1).to(torch.int32)
        s["logit"] = torch.where(there, logit, 0.0)
        s["grad_scale"] = 1.0 / N
    return s


# ---- the plain forms ----

def _plain_top(s):
    c, k = s["case"], s["case"]["k"]
    x = s["logits"].float()
    V = x.shape[1]
    z = x / c["temperature"]
    m = z.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True))).squeeze(1)
    # the k largest, of equal ones the first: those above the k-th largest, and as many of its equals as there is room for
    bar = torch.topk(x, k).values[:, -1:]
    above, equal = x > bar, x == bar
    chosen = above | (equal & (torch.cumsum(equal, 1) <= k - above.sum(1, keepdim=True)))
    at = torch.arange(V, device=DEV, dtype=torch.int32)
    at = -torch.topk(torch.where(chosen, -at, -2 ** 31 + 1), k).values.long()            # the chosen, lowest index first
    best, order = torch.sort(x.gather(1, at), dim=1, descending=True, stable=True)
    return at.gather(1, order).to(torch.int32), best, lse


def _plain_distill(s):
    c, tau = s["case"], s["case"]["temperature"]
    z = s["logits"].float() / tau
    there = s["token"] >= 0
    at = s["token"].clamp(min=0).long()
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    lp = z.gather(1, at) - lse
    listed_ = torch.zeros_like(e).scatter_add_(1, at, there.float()) > 0
    lw = torch.where(there, s["logit"].double() / tau, -math.inf)
    lw = lw - (s["lse"].double()[:, None] if c["rest"] else torch.logsumexp(lw, 1, keepdim=True))
    w = torch.where(there, torch.exp(lw), 0.0)
    lw = torch.where(there, lw, 0.0)
    W = w.sum(1, keepdim=True)
    p = e / total
    g = torch.zeros(1, device=DEV)
    if c["rest"]:
        R = (1.0 - W).clamp(min=LEAST_REST)
        rest = torch.where(listed_, 0.0, e).sum(1, keepdim=True)
        T, lT, lR = rest / total, torch.log(rest) - torch.log(total), torch.log(R).float()
        R = R.float()
        none = rest == 0
    w, lw, W = w.float(), lw.float(), W.float()
    if c["reverse"]:
        ps = torch.where(there, torch.exp(lp), 0.0)
        loss = (ps * (lp - lw)).sum(1, keepdim=True) + torch.where(none, 0.0, T * (lT - lR))
        g = p * (lT - lR - loss)
        inside = ps * (lp - lw - loss)
    else:
        loss = (w * (lw - lp)).sum(1, keepdim=True)
        if c["rest"]:
            loss = loss + torch.where(none, 0.0, R * (lR - lT))
            g = p * torch.where(none, W, W + R - R / T)
            inside = torch.where(none, W, W + R) * torch.exp(lp) - w
        else:
            g = p * (W > 0)
            inside = torch.exp(lp) - w
    scale = s["grad_scale"] / tau
    g = g * scale
    g = g.masked_fill_(listed_, 0.0).scatter_add_(1, at, torch.where(there, inside * scale, 0.0))
    return loss.squeeze(1), lse.squeeze(1), g.to(_type(c))


def _supervised(s):
    tok, coef = s["target"].long(), torch.ones(s["target"].numel(), device=DEV)
    if s["corrected"] is not None:
        hit = s["corrected"] != 0
        tok, coef = torch.where(hit, s["teacher_top1"].long(), tok), torch.where(hit, 1.0, s["advantage"])
    if s["mask"] is not None:
        coef = torch.where(s["mask"] != 0, coef, 0.0)
    return tok, coef


def _plain_linear(s):
    c, tau = s["case"], s["case"]["temperature"]
    h, w = s["hidden"].float(), s["weight"].float()
    tok, coef = _supervised(s)
    z = torch.matmul(h, w.t()) / tau
    m = z.amax(1, keepdim=True)
    p = torch.exp(z - m)
    total = p.sum(1, keepdim=True)
    lp = (z.gather(1, tok[:, None]) - m - torch.log(total)).squeeze(1)
    loss = torch.where(coef != 0, -coef * lp, 0.0)
    if not c["backward"]:
        return loss
    g = p.div_(total)
    g.scatter_add_(1, tok[:, None], torch.full((tok.numel(), 1), -1.0, device=DEV))
    g.mul_((coef * (s["grad_scale"] / tau))[:, None])
    return loss, torch.matmul(g, w).to(BF16), torch.matmul(g.t(), h).to(BF16)


# ---- the library's calls ----

def _own(s):
    import paper_2609_36601_b200 as saki
    c = s["case"]
    if c["op"] == "top":
        out = saki.top_logits(s["logits"], c["k"], temperature=c["temperature"])
        return out["token"], out["logit"], out["lse"]
    if c["op"] == "distill":
        out, dlogits = saki.distill_top(s["logits"], s["token"], s["logit"], s["lse"], reverse=c["reverse"], temperature=c["temperature"],
                                        grad_scale=s["grad_scale"])
        return out["loss"], out["lse"], dlogits
    meta = dict(corrected=s["corrected"], teacher_top1=s["teacher_top1"], advantage=s["advantage"], mask=s["mask"], temperature=c["temperature"])
    out = saki.linear_ce(s["hidden"], s["weight"], s["target"], **meta)
    if not c["backward"]:
        return out["loss"]
    dhidden, dweight = saki.linear_ce_bwd(s["hidden"], s["weight"], s["target"], out["lse"], grad_scale=s["grad_scale"], **meta)
    return out["loss"], dhidden, dweight


def run(state):
    if own:
        return _own(state)
    return {"top": _plain_top, "distill": _plain_distill, "linear": _plain_linear}[state["case"]["op"]](state)


# ---- what a pass cannot do without ----

def work(case):
    N, V = case["N"], case["V"]
    if case["op"] == "linear":
        n, d = N - case["masked"], case["d"]
        if not case["backward"]:
            return {"bytes": 2 * (n * d + V * d) + 8 * N, "flops": 2 * n * d * V}
        return {"bytes": 4 * (n * d + V * d) + 8 * N, "flops": 6 * n * d * V}
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "top":
        return {"bytes": N * V * size + N * (8 * case["k"] + 4), "flops": 3 * N * V}
    return {"bytes": 2 * N * V * size + N * (8 * case["k"] + 12), "flops": 6 * N * V}


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"top": _exact_top, "distill": _exact_distill, "linear": _exact_linear}[case["op"]](case, s)


def _rows(N, V, size=1 << 28):
    step = max(1, size // V)
    return [slice(i, min(N, i + step)) for i in range(0, N, step)]


def _exact_top(case, s):
    lse = [torch.logsumexp(s["logits"][r].to(F64) / case["temperature"], 1) for r in _rows(case["N"], case["V"])]
    return None, None, torch.cat(lse)


def _exact_distill(case, s):
    tau, losses, lses, grads = case["temperature"], [], [], []
    for r in _rows(case["N"], case["V"]):
        logp = torch.log_softmax(s["logits"][r].to(F64) / tau, 1)
        lses.append(torch.logsumexp(s["logits"][r].to(F64) / tau, 1))
        token, n = s["token"][r].long(), logp.shape[0]
        row, col = (token >= 0).nonzero(as_tuple=True)
        v = token[row, col]
        # the teacher's log-weights at their tokens, -inf elsewhere
        t = torch.full_like(logp, -math.inf)
        t[row, v] = s["logit"][r].to(F64)[row, col] / tau
        inside = t > -math.inf
        t = t - (s["lse"][r].to(F64) if case["rest"] else torch.logsumexp(t, 1))[:, None]
        w = torch.where(inside, t.exp(), 0.0)
        mass = w.sum(1)
        out_logp = torch.logsumexp(torch.where(inside, -math.inf, logp), 1)      # log of the student's mass outside
        rest = (1 - mass).clamp(min=LEAST_REST) if case["rest"] else torch.zeros(n, dtype=F64, device=DEV)
        rest = torch.where(out_logp == -math.inf, 0.0, rest)
        p = logp.exp()
        if case["reverse"]:
            ratio = torch.where(inside, logp - t, torch.where(rest > 0, out_logp - rest.log(), 0.0)[:, None])
            loss = (p * torch.where(inside, ratio, 0.0)).sum(1) + torch.where(rest > 0, out_logp.exp() * (out_logp - rest.log()), 0.0)
            grad = p * (ratio - loss[:, None])
        else:
            loss = torch.where(inside, w * (t - logp), 0.0).sum(1) + torch.where(rest > 0, rest * (rest.log() - out_logp), 0.0)
            share = torch.where(rest > 0, rest * (-out_logp).exp(), 0.0)
            grad = p * ((mass + rest)[:, None] - torch.where(inside, 0.0, share[:, None])) - w
        losses.append(loss)
        grads.append(grad * (s["grad_scale"] / tau))
    return torch.cat(losses), torch.cat(lses), torch.cat(grads)


def _exact_linear(case, s):
    tau, w = case["temperature"], s["weight"].to(F64)
    tok, coef = _supervised(s)
    losses, dhidden, dweight = [], [], torch.zeros_like(w) if case["backward"] else None
    for r in _rows(case["N"], case["V"], 1 << 27):
        h = s["hidden"][r].to(F64)
        logp = torch.log_softmax(h @ w.t() / tau, 1)
        i = torch.arange(h.shape[0], device=DEV)
        c = coef[r].to(F64)
        losses.append(torch.where(c != 0, -c * logp[i, tok[r]], 0.0))
        if case["backward"]:
            g = logp.exp_()
            g[i, tok[r]] -= 1.0
            g *= (c * s["grad_scale"] / tau)[:, None]
            dhidden.append(g @ w)
            dweight += g.t() @ h
    if not case["backward"]:
        return torch.cat(losses)
    return torch.cat(losses), torch.cat(dhidden), dweight
