"""Beam selection (saki_beam_select) against the float64 oracle: parents and tokens wherever two keys of the oracle's are not within
rounding of one another, scores to the arithmetic's accuracy.

Tolerances.  A key is score + x / tau - lse; the kernel's lse comes from float32 exponentials: the argument of each is rounded once (2^-24 relative, arguments
up to ~30 that matter, in units of log 2), the exponential is 2^-22 off, and the sum of up to 64 of a thread another 64 * 2^-25 at the most: below 4e-6
together, and far less where the errors differ between elements.  A score is that, rounded to float32 once more (2^-24 relative)."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LSE = 4e-6


def _check(logits, score, n, tau=1.0, finished=None, pad=0):
    out = P.beam_select(logits, score, n, temperature=tau, finished=finished, pad=pad)
    z, s = logits.double().cpu().numpy(), score.double().cpu().numpy()
    f = None if finished is None else finished.cpu().numpy()
    tau32 = float(np.float32(tau))
    parent, token, best, status = O.beam_select(z, s, n, tau32, f, pad)
    wide = O.beam_select(z, s, min(n + 1, z.shape[1] * z.shape[2]), tau32, f, pad)[2]
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert np.array_equal(got["row_status"].reshape(status.shape), status)
    none = best == -np.inf
    assert np.array_equal(np.isneginf(got["score"]), none)
    err = np.abs(got["score"] - np.where(none, 0, best))[~none]
    assert err.size == 0 or np.all(err <= LSE + 2.0 ** -24 * np.abs(best[~none])), err.max()
    # where the key differs from its neighbours' by more than both may be off
    clear = np.ones_like(best, dtype=bool)
    gap = wide[:, :-1] - wide[:, 1:]
    gap = np.where(np.isnan(gap), np.inf, gap)
    same_beam = np.zeros(gap.shape, dtype=bool)            # within a beam the order is exact whatever the lse
    wp = O.beam_select(z, s, wide.shape[1], tau32, f, pad)[0]
    same_beam[:] = wp[:, :-1] == wp[:, 1:]
    # two beams with the same logits and scores have the same keys to the bit: ties between them are exact, too
    tight = (gap <= 2 * LSE) & ~same_beam & (gap > 0)
    clear[:, :tight.shape[1]] &= ~tight[:, :n]
    clear[:, 1:] &= ~tight[:, :n - 1][:, :clear.shape[1] - 1]
    for name, want in (("parent", parent), ("token", token)):
        assert np.array_equal(got[name][clear], want[clear]), name
    assert clear.mean() > 0.9
    P.check()
    return got


def _logits(g, B, W, V, dtype, scale=2.0):
    z = scale * torch.randn((B, W, V), generator=g, device=DEV) - 1.1 * torch.log1p(torch.rand((B, W, V), generator=g, device=DEV) * V)
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,W,V,n,tau", [(1, 1, 2, 1, 1.0), (1, 1, 2, 3, 1.0), (3, 4, 1000, 4, 0.7), (2, 5, 32003, 10, 1.3), (16, 8, 8192, 8, 1.0),
                                         (1, 4, 151936, 4, 1.0), (2, 64, 2049, 64, 1.0), (40, 16, 16385, 32, 1.0), (1, 2, 300000, 64, 2.0)])
def test_matches_the_oracle(dtype, B, W, V, n, tau):
    g = torch.Generator(device=DEV).manual_seed(B * 1000 + V + n)
    z = _logits(g, B, W, V, dtype)
    score = -5 * torch.rand((B, W), generator=g, device=DEV)
    _check(z, score, n, tau)
    fin = (torch.rand((B, W), generator=g, device=DEV) < 0.4).to(torch.uint8)
    _check(z, score, n, tau, fin, pad=V - 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_and_alignment(dtype):
    g = torch.Generator(device=DEV).manual_seed(3)
    wide = _logits(g, 3, 2 * 4, 5003, dtype)
    score = -torch.rand((3, 4), generator=g, device=DEV)
    _check(wide[:, ::2, 1:], score, 6)                    # rows that start anywhere
    _check(wide[:, 1::2, 8:4008], score, 6)
    one = wide[:1].expand(3, 8, 5003)[:, :4]              # the groups share their rows: stride 0
    _check(one, score, 5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_equal_logits_and_equal_beams(dtype):
    """Thousands of equal logits (the list overflows), beams that are copies of one another: ties go to the lower beam and token."""
    z = torch.zeros((2, 3, 20000), dtype=dtype, device=DEV)
    score = torch.zeros((2, 3), device=DEV)
    got = _check(z, score, 8)
    assert got["parent"].tolist() == [[0] * 8] * 2 and got["token"].tolist() == [list(range(8))] * 2
    z[:, :, 17] = -0.0                                    # minus zero is zero
    z[0, 1, 19000:] = 1.0
    got = _check(z, score, 20)
    assert got["parent"][0].tolist() == [1] * 20 and got["token"][0].tolist() == list(range(19000, 19020))
    g = torch.Generator(device=DEV).manual_seed(4)
    z = _logits(g, 2, 1, 9000, dtype).expand(2, 4, 9000).contiguous()
    got = _check(z, score[:, :1].expand(2, 4).contiguous(), 9)
    assert got["parent"][0].tolist() == [0, 1, 2, 3, 0, 1, 2, 3, 0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_and_strange_values(dtype):
    inf = float("inf")
    g = torch.Generator(device=DEV).manual_seed(5)
    z = _logits(g, 6, 3, 4100, dtype)
    score = -torch.rand((6, 3), generator=g, device=DEV)
    z[0] = -inf
    z[0, 1, 4099] = 2.0                                   # one continuation in all
    z[1, 0, 5], z[1, 1, 6], z[1, 2, 7] = inf, float("nan"), -inf
    z[2, :, :] = torch.finfo(dtype).min                   # masks of the type's lowest value
    z[2, 0, 9], z[2, 2, 4000] = 1.0, 1.0
    score[3] = torch.tensor([-inf, 0.5, float("nan")])
    score[4] = inf
    z[5, 0, :4090] = -inf
    got = _check(z, score, 12)
    assert got["row_status"].tolist() == [[0, 0, 0], [8, 8, 0], [0, 0, 0], [0, 0, 8], [8, 8, 8], [0, 0, 0]]
    assert got["token"][0].tolist() == [4099] + [-1] * 11 and got["parent"][4].tolist() == [-1] * 12
    fin = torch.zeros((6, 3), dtype=torch.uint8, device=DEV)
    fin[1] = 1                                            # the logits of finished beams are not looked at
    got = _check(z, score, 3, finished=fin, pad=11)
    assert got["row_status"][1].tolist() == [0, 0, 0] and got["token"][1].tolist() == [11] * 3


def test_flags_are_counted():
    z = torch.full((1, 2, 64), float("nan"), device=DEV)
    P.check()
    P.beam_select(z, torch.zeros(1, 2, device=DEV), 2)
    assert P.check() == 2


def test_wide_rows_and_many_groups():
    """More groups than resident blocks, offsets beyond 32 bits."""
    V, B, W = 151936, 4, 4
    z = torch.empty((8000, 2, V), dtype=torch.bfloat16, device=DEV).as_strided((B, W, V), (4500 * V, 600 * V, 1))     # rows up to 4.6 GB apart
    g = torch.Generator(device=DEV).manual_seed(6)
    z.copy_(_logits(g, B, W, V, torch.bfloat16))
    _check(z, torch.zeros((B, W), device=DEV), 4)
    small = _logits(g, 3000, 2, 64, torch.bfloat16)
    _check(small, -torch.rand((3000, 2), generator=g, device=DEV), 2)


def test_captured_and_on_another_stream():
    g = torch.Generator(device=DEV).manual_seed(7)
    z = _logits(g, 4, 4, 5000, torch.bfloat16)
    score = torch.zeros((4, 4), device=DEV)
    want = P.beam_select(z, score, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = P.beam_select(z, score, 4, stream=s)
    s.synchronize()
    graphs = []
    for _ in range(2):                                    # two captured calls have scratch of their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, P.beam_select(z, score, 4)))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for st, (graph, _) in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for o in (got, *(o for _, o in graphs)):
        assert all(torch.equal(o[k], want[k]) for k in want)


def test_the_binding_refuses():
    z, s = torch.zeros((2, 3, 64), device=DEV), torch.zeros((2, 3), device=DEV)
    for bad in (lambda: P.beam_select(z, s, 0), lambda: P.beam_select(z, s, 65), lambda: P.beam_select(z, s[:1], 2), lambda: P.beam_select(z, s.double(), 2),
                lambda: P.beam_select(z, s, 2, pad=64), lambda: P.beam_select(z.transpose(1, 2), s, 2), lambda: P.beam_select(z, s.cpu(), 2),
                lambda: P.beam_select(z, s, 2, finished=torch.zeros((2, 3), dtype=torch.bool, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: P.beam_select(z.half(), s, 2), lambda: P.beam_select(z, s, 2, temperature=0.0), lambda: P.beam_select(z[:, :, :1], s, 2)):
        with pytest.raises(P.SakiError):
            bad()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tau", [1e-30, 1e-6, 0.25, 2.0, 1e6, 3e38])
def test_temperatures_of_any_size(dtype, tau):
    """Sums whose arguments are huge, tiny or denormal, with -inf among the logits and far from 0."""
    g = torch.Generator(device=DEV).manual_seed(3)
    for shift in (0.0, 1000.0, -3e30, 1e36):
        z = (torch.randn((2, 3, 5000), generator=g, device=DEV) * (1 + abs(shift) * 2.0 ** -6) + shift).to(dtype)
        z[:, :, ::7] = -float("inf")
        score = torch.randn((2, 3), generator=g, device=DEV)
        out = P.beam_select(z, score, 4, temperature=tau)
        assert int(out["row_status"].abs().max()) == 0
        zd, t = z.double(), float(np.float32(tau))
        top = zd.amax(-1, keepdim=True)
        keys = score.double()[..., None] + ((zd - top) / t - torch.log(torch.exp((zd - top) / t).sum(-1, keepdim=True)))
        best = keys.flatten(1).topk(4).values
        # the terms of test_gpu_beam_select: LSE, the stored score's rounding; a constant of few bits (denormal) is off by up to 2^-149 of what it multiplies
        tol = LSE + 2.0 ** -24 * best.abs() + 2.0 ** -148 * float((zd[zd > -float("inf")]).abs().max()) * 2
        fin = best > -3e38
        assert ((out["score"].double() - best).abs() <= tol)[fin].all(), (tau, shift)
    P.check()
