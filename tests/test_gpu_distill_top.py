"""Distillation from a teacher's top logits (saki_distill_top) against the float64 oracle, on the streaming kernel and on the float64 one.

Tolerances.  The log-sum-exp comes from float32 exponentials, each off by 2^-22 and its argument's rounding (2^-24 of at most 60 in base 2, so 4e-6), and
partial sums of a few hundred of them (below 300 2^-24 = 2e-5 at the most, 2e-6 as they fall): 1e-5 is granted, and its rounding.  The loss is a sum of
the list's weights times log-probabilities, each as good as the log-sum-exp, the weights as float32 (2^-24 of each term): 1e-5 (1 + sum of w and of pi) and 2^-22 of the terms' magnitudes.
A probability is off by 2e-5 of itself (as the log-sum-exp is); an element of the gradient is a difference of terms of that kind, (W + R) pi, w and the share of the rest, or pi times the
log-ratios, so it is off by 2e-5 of their magnitudes, in bf16 also by half a step of itself, 2^-8."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _np(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _inputs(N, V, k, dtype, seed, near=False):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = 2.0 * torch.randn((N, V), generator=g, device=DEV) - 1.1 * torch.log1p(torch.rand((N, V), generator=g, device=DEV) * V)
    t = s + 0.1 * torch.randn((N, V), generator=g, device=DEV) if near else 0.8 * s + torch.randn((N, V), generator=g, device=DEV)
    logit, token = torch.topk(t, min(k, V), dim=1)
    if k > V:
        token = torch.cat([token, torch.full((N, k - V), -1, device=DEV)], 1)
        logit = torch.cat([logit, torch.zeros((N, k - V), device=DEV)], 1)
    return s.to(dtype), token.to(torch.int32), logit.contiguous(), t, g


def _check(s, token, logit, lse, reverse, tau=1.0, mask=None, grad_scale=1.0, rows=None, kernel=None, **how):
    out, g = P.distill_top(s, token, logit, lse, reverse=reverse, temperature=tau, mask=mask, grad_scale=grad_scale, **how)
    torch.cuda.synchronize()
    if kernel is not None:
        assert P.last_kernel() == kernel
    rr = slice(None) if rows is None else torch.as_tensor(rows, device=DEV)
    tau32 = float(np.float32(tau))
    pick = lambda t: None if t is None else _np(t[rr])
    s64, tok, lg, tl = pick(s), pick(token), pick(logit), pick(lse)
    ref = O.distill_top(s64, tok, lg, tl, reverse, tau32, pick(mask), grad_scale)
    assert np.array_equal(pick(out["row_status"]).astype(np.uint32), ref["status"])
    ok = ref["status"] == 0
    assert np.all(np.abs(pick(out["lse"]) - ref["lse"]) <= 1e-5 + 2.0 ** -24 * np.abs(ref["lse"]))
    # magnitudes of the loss's and the gradient's terms
    N, V = s64.shape
    loss_mag, grad_mag = np.ones(N), np.zeros((N, V))
    for i in np.flatnonzero(ok):
        with np.errstate(all="ignore"):
            lp = s64[i] / tau32 - ref["lse"][i]
            p = np.exp(lp)
        there = (tok[i] >= 0) & ~np.isneginf(lg[i])
        ids, t = tok[i][there], lg[i][there] / tau32
        if not len(ids) and tl is None:
            continue
        lw = t - (tl[i] if tl is not None else np.log(np.exp(t - t.max()).sum()) + t.max())
        w, outside = np.exp(lw), np.ones(V, dtype=bool)
        outside[ids] = False
        S, R = p[outside].sum(), 0.0 if tl is None else max(1 - w.sum(), 2.0 ** -20)
        lS = np.log(S) if S > 0 else 0.0
        R = R if S > 0 else 0.0
        lR = np.log(R) if R else 0.0
        if reverse:
            loss_mag[i] += (p[ids] * (1 + np.abs(lp[ids]) + np.abs(lw))).sum() + S * (abs(lS) + abs(lR))
            grad_mag[i] = p * (1 + abs(lS) + abs(lR) + loss_mag[i])
            grad_mag[i, ids] = p[ids] * (1 + np.abs(lp[ids]) + np.abs(lw) + loss_mag[i])
        else:
            loss_mag[i] += (w * (1 + np.abs(lw) + np.abs(lp[ids]))).sum() + R * (1 + abs(lR) + abs(lS))
            grad_mag[i] = p * (w.sum() + R + (R / S if R else 0.0))
            grad_mag[i, ids] = p[ids] * (w.sum() + R) + w
    err = np.abs(pick(out["loss"]) - ref["loss"])
    assert np.all(err <= 2e-5 * loss_mag), (err / loss_mag).max()
    if g is not None:
        gg = _np(g[rr])
        err = np.abs(gg - ref["grad"])
        bound = 2e-5 * grad_mag * abs(grad_scale) / tau32 + (2.0 ** -8 if s.dtype == BF16 else 2.0 ** -23) * np.abs(ref["grad"]) + 1e-37
        assert np.all(err <= bound), (err / bound).max()
        assert not gg[~ok].any()
    P.check()
    return out, g, ref


MODES = [(False, False), (True, False), (True, True)]      # with the rest, reverse


@pytest.mark.parametrize("rest,reverse", MODES)
@pytest.mark.parametrize("N,V,k,dtype", [(5, 2, 1, BF16), (5, 2, 2, F32), (7, 9, 4, BF16), (3, 100, 128, F32), (9, 1003, 64, BF16), (160, 4099, 65, BF16), (33, 8192, 16, BF16), (40, 32003, 20, F32),
                                         (310, 32000, 64, BF16), (300, 20480, 33, F32)])
def test_matches_the_oracle(N, V, k, dtype, rest, reverse):
    s, token, logit, t, _ = _inputs(N, V, k, dtype, N + V + k)
    tau = 0.8 if k % 2 else 1.0
    lse = torch.logsumexp(t.double() / tau, 1).float() if rest else None
    rows = list(range(0, N, max(1, N // 10))) + [N - 1]
    _check(s, token, logit, lse, reverse, tau, grad_scale=0.37, rows=rows, kernel=4)
    prev = P.set_kernel(1)
    try:
        _check(s[:12], token[:12], logit[:12], None if lse is None else lse[:12], reverse, tau, grad_scale=0.37, kernel=1)
    finally:
        P.set_kernel(prev)


@pytest.mark.parametrize("V,dtype", [(98304, BF16), (98305, BF16), (106496, BF16), (151936, BF16), (151936, F32), (200001, F32), (524281, BF16)])
@pytest.mark.parametrize("reverse", [False, True])
def test_long_rows(V, dtype, reverse):
    N = 298 if V < 150000 else 152             # rows that follow one another in a block
    s, token, logit, t, _ = _inputs(N, V, 128, dtype, V)
    lse = torch.logsumexp(t, 1)
    del t
    _check(s, token, logit, lse, reverse, rows=[0, 1, 147, 148, 149, N - 1], kernel=4)


@pytest.mark.parametrize("rest,reverse", MODES)
def test_a_student_like_its_teacher(rest, reverse):
    """Nearly all mass on the list: what lies outside must not come from a difference."""
    N, V, k = 24, 5000, 64
    s, token, logit, t, g = _inputs(N, V, k, F32, 3, near=True)
    s.scatter_add_(1, token.long(), torch.full((N, k), 25.0, device=DEV))
    logit = logit + 25.0
    t.scatter_add_(1, token.long(), torch.full((N, k), 25.0, device=DEV))
    lse = torch.logsumexp(t.double(), 1).float() if rest else None
    _, _, ref = _check(s, token, logit, lse, reverse, kernel=4)
    _check(s.to(BF16), token, logit, lse, reverse, kernel=4)


@pytest.mark.parametrize("reverse", [False, True])
def test_a_rest_beyond_float32_goes_to_the_float64_kernel(reverse):
    N, V, k = 20, 3000, 8
    s, token, logit, t, g = _inputs(N, V, k, F32, 4)
    for i, far in ((3, 60.0), (4, 120.0), (5, 400.0)):
        s[i, token[i].long()] += far
    s[6] += 2e7                              # logits whose shifts are no float32
    s[7] -= 3e6
    lse = torch.logsumexp(t, 1)
    _check(s, token, logit, lse, reverse, kernel=4)
    all_of_it = torch.arange(100, device=DEV, dtype=torch.int32).repeat(N, 1)
    _check(s[:, :100].contiguous(), all_of_it, t[:, :100].contiguous(), torch.logsumexp(t[:, :100], 1), reverse)      # nothing outside


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rest,reverse", MODES)
def test_masked_and_strange_values(dtype, rest, reverse):
    inf = float("inf")
    N, V, k = 30, 40000, 32
    s, token, logit, t, g = _inputs(N, V, k, dtype, 5)
    lse = torch.logsumexp(t, 1) if rest else None
    low = torch.finfo(dtype).min
    listed = torch.zeros((N, V), dtype=torch.bool, device=DEV).scatter_(1, token.long(), True)
    mask = torch.ones(N, dtype=torch.uint8, device=DEV)
    token[0] = -1                                        # nothing there
    logit[1] = -inf
    token[2, 5:], logit[2, 5:] = -1, float("nan")        # what is not there is not looked at
    s[3] = torch.where(listed[3], s[3], -inf)            # all but the list masked
    s[4] = torch.where(listed[4], s[4], low)
    s[5, :39000] = torch.where(listed[5, :39000], s[5, :39000], -inf)
    s[6, :39000] = torch.where(listed[6, :39000], s[6, :39000], low)
    s[7, :39000] = torch.where(listed[7, :39000], s[7, :39000], -1e9)
    s[8, 1000:] = torch.where(listed[8, 1000:], s[8, 1000:], -1e30)
    s[9, token[9, 3].long()] = -inf                      # listed and masked: flagged
    s[10] = -inf
    s[11, 77] = float("nan")
    s[12, 39999] = inf
    token[13, 7] = V
    token[14, 7] = -2
    token[15, 9] = token[15, 30]                         # twice
    logit[16, 3] = float("nan")
    logit[17, 31] = inf
    mask[18] = 0
    s[18] = float("nan")
    token[18, 0] = V + 5
    if rest:
        lse[19], lse[20] = inf, float("nan")
        lse[21] -= 3.0                                   # a list that says more than there is: R at its least
    s[22] = 0.0                                          # all equal
    s[23, token[23].long()] = low                        # listed, at the lowest value
    if reverse:
        s[23] = 0.0
    s[24] = torch.where(torch.arange(V, device=DEV) == token[24, 0], 50.0, -50.0).to(dtype)
    P.check()
    out, _ = P.distill_top(s, token, logit, lse, reverse=reverse, mask=mask)
    flags = out["row_status"].cpu().numpy()
    assert flags[9:19].tolist() == [8, 8, 8, 8, 16, 16, 16, 8, 8, 4]
    assert P.check() == 9 + (2 if rest else 0)
    finite = [i for i in range(N) if i != 23]            # (a listed token at the type's lowest value has a loss of 1e38 and more)
    _check(s, token, logit, lse, reverse, mask=mask, rows=finite, kernel=4)
    prev = P.set_kernel(1)
    try:
        _check(s, token, logit, lse, reverse, mask=mask, rows=finite, kernel=1)
    finally:
        P.set_kernel(prev)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignment(dtype):
    N, V, k = 21, 3001, 10
    s, token, logit, t, g = _inputs(N, V, k, dtype, 6)
    lse = torch.logsumexp(t, 1)
    base, gbase, _ = _check(s, token, logit, lse, False)
    wide = torch.full((N, V + 37), float("nan"), dtype=dtype, device=DEV)
    tw, lw = torch.full((N, k + 3), -7, dtype=torch.int32, device=DEV), torch.full((N, k + 3), float("nan"), device=DEV)
    tw[:, 1:1 + k], lw[:, 1:1 + k] = token, logit
    for off in (0, 1, 3, 8, 37):
        view = wide[:, off:off + V]
        view.copy_(s)
        into = torch.full((N, V + 11), 7.0, dtype=dtype, device=DEV)
        out, grad, _ = _check(view, tw[:, 1:1 + k], lw[:, 1:1 + k], lse, False, dlogits=into[:, 2:2 + V])
        assert (into[:, :2] == 7).all() and (into[:, 2 + V:] == 7).all()      # nothing beside the rows
        same = torch.full_like(wide, 7.0)
        _check(view, token, logit, lse, False, dlogits=same[:, off:off + V])      # lies like the rows
        assert (same[:, :off] == 7).all() and (same[:, off + V:] == 7).all()
        wide.fill_(float("nan"))
    with pytest.raises(P.SakiError, match="row stride"):  # every row the same memory
        P.distill_top(s[:1].expand(N, V), token, logit, lse, dlogits=torch.empty_like(s))
    _check(s, token, logit, lse, True, dlogits=None)
    empty, ge = P.distill_top(s[:0], token[:0], logit[:0])
    assert empty["loss"].numel() == 0 and ge.shape == (0, V)


@pytest.mark.parametrize("reverse", [False, True])
def test_rows_too_long_for_the_streaming_kernel(reverse):
    N, V = 3, 300001
    s, token, logit, t, _ = _inputs(N, V, 40, F32, 10)
    _check(s, token, logit, torch.logsumexp(t, 1), reverse, kernel=1)


def test_offsets_beyond_32_bits():
    V, N = 151936, 5
    s = torch.empty(4 * 5_000_000_00 + V, dtype=BF16, device=DEV).as_strided((N, V), (500_000_000, 1))
    x, token, logit, t, g = _inputs(N, V, 16, BF16, 7)
    s.copy_(x)
    _check(s, token, logit, torch.logsumexp(t, 1), False, dlogits=torch.empty((N, V), dtype=BF16, device=DEV))


@pytest.mark.parametrize("rest,reverse", MODES)
def test_the_gradient_against_differences(rest, reverse):
    N, V, k = 16, 700, 12
    s, token, logit, t, g = _inputs(N, V, k, F32, 8)
    lse = torch.logsumexp(t, 1) if rest else None
    _, grad = P.distill_top(s, token, logit, lse, reverse=reverse)
    for _ in range(4):
        step = torch.randn((N, V), generator=g, device=DEV) * 0.02
        f = [P.distill_top(s + d, token, logit, lse, reverse=reverse, dlogits=None)[0]["loss"].double() for d in (step, -step)]
        move = (s + step).double() - (s - step).double()
        want = (grad.double() * move).sum(1)
        # third derivatives are below a few times the cube of the steps (the log-ratios, up to 30 here, times it for the reverse divergence); losses to 2e-5
        bound = 30 * (4 * 0.02) ** 3 * 8 / 6 + 1e-4
        assert bool(((f[0] - f[1] - want).abs() <= bound).all()), (f[0] - f[1] - want).abs().max()


def test_captured_and_on_another_stream():
    s, token, logit, t, g = _inputs(64, 32003, 50, BF16, 9)
    lse = torch.logsumexp(t, 1)
    out, grad = P.distill_top(s, token, logit, lse)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    o2, g2 = P.distill_top(s, token, logit, lse, stream=other)
    other.synchronize()
    assert torch.equal(o2["loss"], out["loss"]) and torch.equal(g2, grad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o3, g3 = P.distill_top(s, token, logit, lse)
    for _ in range(2):
        g3.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o3["loss"], out["loss"]) and torch.equal(g3, grad)
