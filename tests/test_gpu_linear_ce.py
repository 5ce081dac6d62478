"""Cross entropy from hidden states (saki_linear_ce_fwd, saki_linear_ce_bwd) against the float64 oracle.

Tolerances.  A logit is a float32 sum of d exact products: off by at most d 2^-23 of the sum of their magnitudes (the tensor cores may cut
instead of rounding: a whole step an addition); scaling and the exponential's argument add 2^-23 of the argument.  The log-sum-exp and the log-probability
are off by as much as the logits, and by the exponentials and their sums (4e-6, rounding to float32 2^-24).  A probability is off by that
share of itself, twice (logit and log-sum-exp); the supervised element of G is the difference pi - 1, so it is off by that share of pi, however little is left of the
difference: a gradient by that share of the sum of its terms with pi in G's place.  G is rounded to bf16, 2^-8 of each element; its products are summed in float32
(K 2^-23 of the sum of the terms' magnitudes), and the sum is rounded to bf16, 2^-8 of itself."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _np(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def _inputs(N, d, V, seed, lean=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = (2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device=DEV)).to(BF16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn((N, d), generator=g, device=DEV) + lean * torch.rand((N, 1), generator=g, device=DEV) * w[target.long()].float()).to(BF16)
    return h, w, target, g


def _check(h, w, target, tau=1.0, grad_scale=1.0, advantage=None, corrected=None, teacher_top1=None, mask=None, rollout_status=None, **how):
    meta = dict(advantage=advantage, corrected=corrected, teacher_top1=teacher_top1, mask=mask, rollout_status=rollout_status)
    out = P.linear_ce(h, w, target, temperature=tau, **meta)
    dh, dw = P.linear_ce_bwd(h, w, target, out["lse"], temperature=tau, grad_scale=grad_scale, **meta, **how)
    torch.cuda.synchronize()
    tau32 = float(np.float32(tau))
    h64, w64 = _np(h), _np(w)
    rows = O.supervised(w.shape[0], _np(target), **{k: _np(v) for k, v in meta.items()})
    with np.errstate(all="ignore"):
        mags = (np.abs(h64) @ np.abs(w64).T / tau32).max(axis=1)
    z_err = np.where(np.isfinite(mags) & [t >= 0 for t, _, _ in rows], (h.shape[1] + 4) * 2.0 ** -23 * mags + 4e-6, 0.0)
    ref = O.linear_ce(h64, w64, rows, tau32, grad_scale, 2 * z_err)
    assert np.array_equal(_np(out["row_status"]).astype(np.uint32), ref["status"])
    ok = np.isfinite(ref["lse"])
    assert np.array_equal(np.isfinite(_np(out["lse"])), ok)
    coef = np.array([c for _, c, _ in rows])
    for name, scale in (("lse", 1.0), ("logp_tok", 1.0), ("loss", np.abs(coef))):
        err = np.abs(_np(out[name]) - ref[name])[ok]
        assert np.all(err <= ((2 * z_err + 2.0 ** -22 * (np.abs(ref["lse"]) + np.abs(ref["logp_tok"]))) * scale)[ok]), (name, err.max())
    for got, name, K in ((dh, "dhidden", w.shape[0]), (dw, "dweight", h.shape[0])):
        if got is None:
            continue
        want, mag = ref[name], ref[name + "_abs"]
        err = np.abs(_np(got) - want)
        bound = (2.0 ** -8 + K * 2.0 ** -23) * mag + ref[name + "_p"] + 2.0 ** -8 * np.abs(want) + 1e-30
        assert np.all(err <= bound), (name, (err / bound).max())
    P.check()
    return out, dh, dw, ref


@pytest.mark.parametrize("N,d,V,tau", [(1, 8, 2, 1.0), (3, 64, 7, 0.7), (200, 64, 4128, 1.0), (131, 96, 1003, 1.3), (257, 256, 8192, 1.0), (128, 8, 256, 1.0),
                                        (600, 520, 3301, 1.0), (65, 1096, 32003, 1.1), (513, 264, 511, 1.0)])
def test_matches_the_oracle(N, d, V, tau):
    h, w, target, _ = _inputs(N, d, V, 7 * N + d)
    _check(h, w, target, tau, grad_scale=0.37)


def _meta(N, V, g):
    return dict(corrected=(torch.rand(N, generator=g, device=DEV) < 0.3).to(torch.uint8), teacher_top1=torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32),
                advantage=torch.randn(N, generator=g, device=DEV), mask=(torch.rand(N, generator=g, device=DEV) < 0.6).to(torch.uint8))


@pytest.mark.parametrize("N,d,V", [(300, 128, 2000), (777, 72, 5003)])
def test_routing_metadata(N, d, V):
    h, w, target, g = _inputs(N, d, V, N)
    _check(h, w, target, grad_scale=1.0 / N, **_meta(N, V, g))


def test_rows_that_contribute_nothing_reach_nothing():
    """Masked and flagged rows may hold anything: NaN and infinities in their hidden states reach no gradient."""
    N, d, V = 300, 64, 1000
    h, w, target, g = _inputs(N, d, V, 5)
    meta = _meta(N, V, g)
    status = torch.zeros(N, dtype=torch.int32, device=DEV)
    meta["mask"][:8] = torch.tensor([0, 1, 1, 1, 1, 1, 1, 1], dtype=torch.uint8)
    meta["corrected"][:8] = torch.tensor([0, 0, 1, 0, 0, 0, 1, 0], dtype=torch.uint8)
    h[0] = float("nan")
    status[1] = 64
    h[1, 3] = float("inf")
    meta["teacher_top1"][2] = V
    h[2, 1] = -float("inf")
    target[3] = -1
    meta["advantage"][4] = float("nan")
    h[5, 7] = float("nan")                    # contributes, and is not finite: flagged by its own log-sum-exp
    meta["advantage"][6] = float("inf")       # corrected: not read
    h[7] = 1e30                               # logits of about 1e31
    P.check()
    out, dh, dw, ref = _check(h, w, target, rollout_status=status, grad_scale=0.1, **meta)
    assert _np(out["row_status"])[:7].tolist() == [4, 64, 16, 16, 8, 8, 0]
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all() and not dh[:6].any()
    P.linear_ce(h, w, target, rollout_status=status, **meta)
    assert P.check() == 4
    none = P.linear_ce(h, w, target, mask=torch.zeros(N, dtype=torch.uint8, device=DEV))
    assert not none["loss"].any() and (none["row_status"] == 4).all()
    dh, dw = P.linear_ce_bwd(h, w, target, none["lse"], mask=torch.zeros(N, dtype=torch.uint8, device=DEV), dweight=torch.full_like(w, float("nan")))
    assert not dh.any() and not dw.any()      # no row at all


def test_a_weight_that_is_not_finite():
    h, w, target, _ = _inputs(70, 64, 300, 6)
    w[17, 3] = float("nan")
    out, dh, dw, _ = _check(h, w, target)
    assert (out["row_status"] == 8).all() and not dh.any() and not dw.any()
    P.check()


def test_strides_and_alignment():
    N, d, V = 150, 72, 700
    h, w, target, g = _inputs(N, d, V, 8)
    wide_h, wide_w = torch.zeros((N, d + 13), dtype=BF16, device=DEV), torch.zeros((V, d + 16), dtype=BF16, device=DEV)
    wide_h[:, 3:3 + d], wide_w[:, 8:8 + d] = h, w
    a = _check(h, w, target)
    dh, dw = torch.full((N, d + 8), 7.0, dtype=BF16, device=DEV), torch.full((V, d + 24), 7.0, dtype=BF16, device=DEV)
    b = _check(wide_h[:, 3:3 + d], wide_w[:, 8:8 + d], target, dhidden=dh[:, 8:], dweight=dw[:, 16:16 + d])
    for x, y in zip(a[:3], b[:3]):
        for k in (x if isinstance(x, dict) else [None]):
            assert torch.equal(x[k], y[k]) if k else torch.equal(x, y)
    assert (dh[:, :8] == 7).all() and (dw[:, :16] == 7).all() and (dw[:, 16 + d:] == 7).all()


def test_one_gradient_alone_and_no_rows():
    h, w, target, _ = _inputs(90, 64, 900, 9)
    _, dh, dw, _ = _check(h, w, target)
    assert torch.equal(_check(h, w, target, dweight=None)[1], dh) and torch.equal(_check(h, w, target, dhidden=None)[2], dw)
    none = P.linear_ce(h[:0], w, target[:0])
    assert none["loss"].numel() == 0
    dh, dw = P.linear_ce_bwd(h[:0], w, target[:0], none["lse"], dweight=torch.full_like(w, 3.0))
    assert dh.numel() == 0 and not dw.any()


@pytest.mark.parametrize("N,d,V,rows", [(2300, 136, 40000, 12), (300, 2560, 151936, 6)])
def test_pieces_and_parts(N, d, V, rows):
    """Vocabularies of several pieces, sums cut into parts: some rows of each gradient against float64 products on the GPU."""
    h, w, target, g = _inputs(N, d, V, N + d)
    mask = (torch.rand(N, generator=g, device=DEV) < 0.8).to(torch.uint8)
    out = P.linear_ce(h, w, target, mask=mask)
    dh, dw = P.linear_ce_bwd(h, w, target, out["lse"], mask=mask)
    G = torch.empty((N, V), dtype=torch.float64, device=DEV)
    w64 = w.double()
    z_err = (d + 4) * 2.0 ** -23 * float((h.double().abs() @ w64.abs().t()).max()) + 4e-6
    for i in range(0, N, 256):
        logp = torch.log_softmax(h[i:i + 256].double() @ w64.t(), 1)
        p = logp.exp()
        r = torch.arange(p.shape[0], device=DEV)
        assert float((out["loss"][i:i + 256].double() + logp[r, target[i:i + 256].long()] * mask[i:i + 256]).abs().max()) <= 2 * z_err + 1e-5
        p[r, target[i:i + 256].long()] -= 1.0
        G[i:i + 256] = p * mask[i:i + 256, None]
    want = G @ w64
    mag = torch.empty_like(want)
    for i in range(0, N, 256):
        mag[i:i + 256] = G[i:i + 256].abs() @ w64.abs()
    assert bool(((dh.double() - want).abs() <= (2.0 ** -8 + V * 2.0 ** -23 + 2 * z_err) * mag + 2.0 ** -8 * want.abs()).all())
    h64 = torch.where(mask[:, None] != 0, h.double(), 0.0)
    want = G.t() @ h64
    mag = G.abs().t() @ h64.abs()
    assert bool(((dw.double() - want).abs() <= (2.0 ** -8 + N * 2.0 ** -23 + 2 * z_err) * mag + 2.0 ** -8 * want.abs()).all())


@pytest.mark.parametrize("N,d,V", [((1 << 20) + 100, 2112, 300), (40, 2112, (1 << 20) + 77)])
def test_offsets_beyond_32_bits(N, d, V):
    """Hidden states, or weights, of more than 2^32 bytes: all of the loss and of both gradients against float64 products on the GPU, in blocks."""
    h, w, target, g = _inputs(N, d, V, 31)
    out = P.linear_ce(h, w, target)
    dh, dw = P.linear_ce_bwd(h, w, target, out["lse"])
    rows, cols = 1 << 14, 1 << 14
    z_err = 0.0
    for i in range(0, N, rows):
        hi = h[i:i + rows].double()
        yi = target[i:i + rows].long()
        lse = torch.full((hi.shape[0],), -float("inf"), dtype=torch.float64, device=DEV)
        for j in range(0, V, cols):
            wj = w[j:j + cols].double()
            lse = torch.logaddexp(lse, torch.logsumexp(hi @ wj.t(), 1))
            z_err = max(z_err, (d + 4) * 2.0 ** -23 * float((hi.abs() @ wj.abs().t()).max()) + 4e-6)
        tol = 2 * z_err + 2.0 ** -22 * 2 * float(lse.abs().max())
        z_tok = (hi * w[yi].double()).sum(1)
        assert float((out["loss"][i:i + rows].double() - (lse - z_tok)).abs().max()) <= tol
        want, mag = torch.zeros_like(hi), torch.zeros_like(hi)
        if i == 0 and N > rows:
            dw_want, dw_mag = ([torch.zeros((min(cols, V - j), d), dtype=torch.float64, device=DEV) for j in range(0, V, cols)] for _ in range(2))
        for b, j in enumerate(range(0, V, cols)):
            wj = w[j:j + cols].double()
            G = torch.exp(hi @ wj.t() - lse[:, None])
            here = (yi >= j) & (yi < j + wj.shape[0])
            p_tok = torch.exp(z_tok - lse)
            G[here.nonzero()[:, 0], yi[here] - j] -= 1.0
            a = G.abs()
            a[here.nonzero()[:, 0], yi[here] - j] += p_tok[here] * 2 * tol / 2.0 ** -8      # (pi - 1 is off by a share of pi)
            want += G @ wj
            mag += a @ wj.abs()
            if N <= rows:                     # (one block of rows: there and then)
                x, m = G.t() @ hi, a.t() @ hi.abs()
                assert bool(((dw[j:j + cols].double() - x).abs() <= (2.0 ** -8 + N * 2.0 ** -23 + 2 * tol) * m + 2.0 ** -8 * x.abs() + 1e-30).all()), j
            else:
                dw_want[b] += G.t() @ hi
                dw_mag[b] += a.t() @ hi.abs()
        assert bool(((dh[i:i + rows].double() - want).abs() <= (2.0 ** -8 + V * 2.0 ** -23 + 2 * tol) * mag + 2.0 ** -8 * want.abs()).all()), i
    if N > rows:
        for b, j in enumerate(range(0, V, cols)):
            assert bool(((dw[j:j + cols].double() - dw_want[b]).abs() <= (2.0 ** -8 + N * 2.0 ** -23 + 2 * tol) * dw_mag[b] + 2.0 ** -8 * dw_want[b].abs()).all())


def test_losses_next_to_zero():
    """Confident rows with logits of hundreds: the loss comes from differences to the largest logit.  What is left is the sum of a row, 1 and little more: at most some 18 additions to
    the 1 in float32, 2^-24 each, and the exponentials' own share of what the others have."""
    N, d, V = 300, 64, 5000
    g = torch.Generator(device=DEV).manual_seed(30)
    w = (2.0 / d ** 0.5 * torch.randn((V, d), generator=g, device=DEV)).to(BF16)
    target = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.linspace(5, 100, N, device=DEV)[:, None] * w[target.long()].float()).to(BF16)
    out = P.linear_ce(h, w, target)
    z = h.double() @ w.double().t()
    top = z.gather(1, target.long()[:, None])
    others = torch.exp(z - top).scatter_(1, target.long()[:, None], 0.0).sum(1)
    assert float(top.max()) > 300 and bool((z.amax(1, keepdim=True) == top).all())
    z_err = (d + 4) * 2.0 ** -23 * (h.double().abs() @ w.double().abs().t()).amax(1) + 4e-6
    want = torch.log1p(others)
    assert bool(((out["loss"].double() - want).abs() <= 18 * 2.0 ** -24 + 2 * z_err * others).all())


def test_the_gradient_against_differences():
    """Central differences of the loss (float64 sum of the float32 losses) in random directions of bf16 steps."""
    N, d, V = 64, 64, 500
    h, w, target, g = _inputs(N, d, V, 21)
    out = P.linear_ce(h, w, target)
    dh, dw = P.linear_ce_bwd(h, w, target, out["lse"])
    for x, grad in ((h, dh), (w, dw)):
        for _ in range(3):
            step = 0.03 * torch.randn(x.shape, generator=g, device=DEV)
            up, down = (x.float() + step).to(BF16), (x.float() - step).to(BF16)
            f = [float(P.linear_ce(y if x is h else h, y if x is w else w, target)["loss"].double().sum()) for y in (up, down)]
            move = up.double() - down.double()
            want = float((grad.double() * move).sum())
            # third derivatives of a log-sum-exp are below 2 spread^3 of the logits' steps; and what the gradient's roundings make, 2^-8 of its terms
            dz = (move / 2 @ w.double().t() if x is h else h.double() @ (move / 2).t()).abs().amax(1)
            bound = float((4 / 3 * dz ** 3).sum()) + 2.0 ** -7 * float((grad.double() * move).abs().sum()) + N * 2e-5
            assert abs(f[0] - f[1] - want) <= bound, (f, want, bound)


def test_captured_and_on_another_stream():
    h, w, target, _ = _inputs(300, 128, 5000, 22)
    out = P.linear_ce(h, w, target)
    want = (out["loss"], *P.linear_ce_bwd(h, w, target, out["lse"]))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    o = P.linear_ce(h, w, target, stream=other)
    got = (o["loss"], *P.linear_ce_bwd(h, w, target, o["lse"], stream=other))
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = P.linear_ce(h, w, target)
        got = (o["loss"], *P.linear_ce_bwd(h, w, target, o["lse"]))
    for _ in range(2):
        for t in got:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    h.mul_(0.5)                               # a replay reads what is there by then
    graph.replay()
    o = P.linear_ce(h, w, target)
    torch.cuda.synchronize()
    assert torch.equal(got[0], o["loss"]) and not torch.equal(got[0], want[0])


def test_the_same_call_gives_the_same_bits():
    h, w, target, _ = _inputs(700, 264, 9000, 23)
    first = None
    for _ in range(4):
        out = P.linear_ce(h, w, target)
        got = (out["loss"], out["lse"], *P.linear_ce_bwd(h, w, target, out["lse"]))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))
