"""A row's top logits and log-sum-exp (saki_top_logits) against the float64 oracle: tokens and logits exactly, the log-sum-exp to what float32 exponentials give.

Tolerance of the log-sum-exp.  An exponential is off by 2^-22 and its argument's rounding (at most 60 in base 2: 4e-6 as 2^-24 of it); a thread's partial sums of at most 160 pairs
another 160 2^-24 = 1e-5 if all went one way: 1e-5 is granted, and the rounding of the result, 2^-24 of it."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _check(x, k, tau=1.0, rows=None, out=None):
    out = P.top_logits(x, k, temperature=tau) if out is None else out
    torch.cuda.synchronize()
    rr = slice(None) if rows is None else torch.as_tensor(rows, device=DEV)
    token, logit, lse, status = O.top_logits(x[rr].double().cpu().numpy(), k, float(np.float32(tau)))
    got = {n: v[rr].cpu().numpy() for n, v in out.items()}
    assert np.array_equal(got["row_status"].astype(np.uint32), status)
    assert np.array_equal(got["token"], token)
    assert np.array_equal(got["logit"].astype(np.float64), logit)
    same = np.isneginf(lse) & np.isneginf(got["lse"])
    with np.errstate(invalid="ignore"):
        assert np.all(same | (np.abs(got["lse"] - lse) <= 1e-5 + 2.0 ** -24 * np.abs(lse))), np.nanmax(np.abs(got["lse"] - lse))
    P.check()
    return out


def _logits(N, V, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (2.0 * torch.randn((N, V), generator=g, device=DEV) - 1.1 * torch.log1p(torch.rand((N, V), generator=g, device=DEV) * V)).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,V,k,tau", [(1, 2, 1, 1.0), (3, 2, 5, 0.7), (5, 9, 9, 1.0), (2, 100, 128, 1.0), (9, 1003, 64, 1.3), (40, 4099, 128, 1.0), (300, 2048, 1, 1.0), (8, 151936, 64, 1.0),
                                        (1, 151936, 128, 0.5), (330, 32003, 100, 1.25), (320, 40961, 7, 1.0), (3, 163841, 50, 1.0), (2, 1000000, 128, 1.0)])
def test_matches_the_oracle(N, V, k, tau, dtype):
    rows = None if N < 20 else list(range(0, N, N // 10)) + [N - 1]
    _check(_logits(N, V, dtype, N + V + k), k, tau, rows)


@pytest.mark.parametrize("V", [20481, 32003, 65536, 65537])
@pytest.mark.parametrize("N", [740, 800, 1500])
def test_float32_rows_about_whole_rounds_of_blocks(N, V):
    x = _logits(N, V, F32, N + V)
    x[1], x[2, ::3] = torch.linspace(-8, 8, V, device=DEV), -float("inf")      # all that is best in a stretch; masks
    _check(x, 100, rows=[0, 1, 2, N // 2, N - 1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_long_rows(dtype):
    x = _logits(600, 163840, dtype, 1)        # the longest that one block takes whole
    _check(x, 128, rows=[0, 1, 299, 598, 599])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [1, 400])
def test_orders_that_are_hard(dtype, N):
    """Sorted rows (all that is best in few threads' pieces or in one stretch), equal ones, two values, masks: lists overflow or fall short."""
    V, k, inf = 30000, 100, float("inf")
    up = torch.linspace(-8, 8, V, device=DEV)
    rows = [up, up.flip(0), torch.zeros(V, device=DEV), torch.full((V,), torch.finfo(dtype).min, device=DEV), torch.full((V,), -inf, device=DEV),
            torch.where(torch.arange(V, device=DEV) % 3000 == 7, 2.0, torch.finfo(dtype).min), torch.where(torch.arange(V, device=DEV) % 3000 == 7, 2.0, -inf),
            torch.where(torch.arange(V, device=DEV) % 2 == 0, 1.0, -0.0), torch.where(torch.arange(V, device=DEV) < 700, 5.0, up / 100),
            torch.where(torch.arange(V, device=DEV) // 8 % 256 == 77, up + 20, up), torch.where(torch.arange(V, device=DEV) == V - 1, -3.0, -inf),
            torch.full((V,), -1e9, device=DEV), torch.where(torch.arange(V, device=DEV) >= 29000, up, -1e9), torch.where(torch.arange(V, device=DEV) >= 29000, up, -1e30), up * 1e6, up * 1e30]
    x = torch.stack(rows).to(dtype)
    x = x.repeat((N + len(rows) - 1) // len(rows), 1) if N > 1 else x
    out = _check(x, k, rows=list(range(len(rows))))
    if N > 1:
        for name, v in out.items():
            v = v.view(-1, len(rows), *v.shape[1:])
            assert torch.equal(v, v[:1].expand_as(v)), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [4, 500])
def test_values_that_are_not_finite(dtype, N):
    inf = float("inf")
    x = _logits(N, 20011, dtype, 2)
    x[0, 20010], x[1, 0], x[2, 5000:5300] = inf, float("nan"), float("nan")
    if N > 4:
        x[5] = float("nan")
        x[6, ::2] = -float("nan")
        x[7, 3] = -inf
    P.check()
    out = P.top_logits(x, 12)
    flags = 3 if N == 4 else 5
    assert int((out["row_status"] == 8).sum()) == flags == P.check()
    _check(x, 12, rows=list(range(4 if N == 4 else 10)))
    tiny = P.top_logits(x[3:4], 3, temperature=1e-30)      # the largest alone has any weight
    assert abs(float(tiny["lse"]) / float(tiny["logit"][0, 0]) * 1e-30 - 1) < 1e-6


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignment(dtype):
    wide = _logits(11, 7001, dtype, 3)
    for off in (0, 1, 3, 6, 8):
        _check(wide[:, off:off + 6007], 33)
        _check(wide[::2, off:off + 6007], 33)
    _check(wide[:1, 1:].expand(300, 7000), 20, rows=[0, 299])      # every row the same memory
    assert P.top_logits(wide[:0], 4)["token"].shape == (0, 4)


def test_offsets_beyond_32_bits():
    V, N = 151936, 5
    x = torch.empty(4 * 500_000_000 + V, dtype=BF16, device=DEV).as_strided((N, V), (500_000_000, 1))
    x.copy_(_logits(N, V, BF16, 4))
    _check(x, 64)


def test_captured_and_on_another_stream():
    for N in (6, 400):
        x = _logits(N, 32000, BF16, 5)
        want = P.top_logits(x, 40)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        got = P.top_logits(x, 40, stream=other)
        other.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = P.top_logits(x, 40)
        for _ in range(2):
            for v in got.values():
                v.fill_(0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(got[n], want[n]) for n in want)
