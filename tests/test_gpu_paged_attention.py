"""Attention over a paged cache (saki_paged_attention) against the float64 oracle.

Tolerances, per row, with A = sum_x w_x |v_x| (weights w of the oracle's) and S = scale * max_x sum_d |q_d k_xd|:
  a score is a float32 sum of D products (the tensor cores may cut where they add, 2^-23 a step), scaled by a rounded constant and subtracted from the maximum:
  off by at most e = (D + 4) 2^-23 S; the exponential is 2^-22 off; so a weight is off by a share of e + 2^-21, and, in two bf16 terms, 2^-16 more;
  sums over n positions add n 2^-23.  Each of it enters the output twice (numerator, denominator), times A; the stored value is rounded once more,
  by eps / 2 relative to itself.  lse: e + 2^-21 + n 2^-23, and its own rounding."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


def _make(B, Q, H, G, D, page, lengths, dtype, seed, head_major=False, extra=3, fill=None):
    """q, pools and tables; slots that hold no position are `fill` (default: numbers like the others)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    counts = [-(-n // page) for n in lengths]
    max_pages, n_pages = max(1, max(counts)) + extra, sum(counts) + 4
    shape = (n_pages, H, page, D) if head_major else (n_pages, page, H, D)
    pools = [torch.randn(shape, generator=g, device=DEV).to(dtype) for _ in range(2)]
    if head_major:
        pools = [p.transpose(1, 2) for p in pools]
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    used = torch.zeros((n_pages, page), dtype=torch.bool)
    for b, (n, c) in enumerate(zip(lengths, counts)):
        for x in range(c):
            table[b, x] = ids.pop()
            used[table[b, x], :min(page, n - x * page)] = True
    if fill is not None:
        for p in pools:
            p[~used.to(DEV)] = fill
    q = (2 * torch.randn((B, Q, H * G, D), generator=g, device=DEV)).to(dtype)
    return q, pools[0], pools[1], table.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV)


def _np(t):
    return t.detach().cpu().double().numpy()


def _check(q, k, v, table, length, scale=None, window=0, sinks=0, n_query=None, out=None, got=None, rows=None):
    D = q.shape[3]
    sc = 1 / np.sqrt(D) if scale is None else scale
    if got is None:
        got = P.paged_attention(q, k, v, table, length, scale=scale, window=window, sinks=sinks, n_query=n_query, out=out)
    nq = None if n_query is None else n_query.cpu().numpy()
    args = (table.cpu().numpy(), length.cpu().numpy(), float(np.float32(sc)), nq, window, sinks)
    qn, kn, vn = _np(q), np.nan_to_num(_np(k), posinf=0, neginf=0), _np(v)
    want, lse, status = O.paged_attention(_np(q), _np(k), vn, *args)
    size, _, _ = O.paged_attention(_np(q), kn, np.nan_to_num(np.abs(vn), posinf=0), *args)
    bound = abs(float(sc)) * np.sqrt((qn ** 2).sum(-1)) * np.sqrt((kn ** 2).sum(-1).max())      # |q||k| >= sum |q_d k_d|
    n = int(length.clamp(min=0).max())
    e = (D + 4) * 2.0 ** -23 * bound
    half = torch.finfo(q.dtype).eps / 2
    share = 2 * (e + 2.0 ** -21 + (2.0 ** -16 if q.dtype == BF16 else 0) + n * 2.0 ** -23)
    o, L, st = (_np(t) for t in got)
    assert np.array_equal(st, status)
    where = np.isfinite(want)
    assert np.array_equal(np.isfinite(o), where)
    err = np.abs(o - np.where(where, want, 0))
    tol = (half * (1 + share[..., None]) * np.abs(want) + share[..., None] * size)
    assert np.all((err <= tol + 1e-30)[where]), (err - tol)[where].max()
    there = lse > -np.inf
    assert np.array_equal(np.isneginf(L), lse == -np.inf)
    fin = np.isfinite(lse)
    assert np.array_equal(np.isfinite(L), fin) and np.array_equal(np.isnan(L), np.isnan(lse) & ~there | np.isnan(lse))
    assert np.all((np.abs(L - np.where(fin, lse, 0)) <= e + 2.0 ** -21 + n * 2.0 ** -23 + 2.0 ** -22 * np.abs(lse))[fin])
    return got


CASES = [  # B, Q, H, G, D, page, lengths
    (1, 1, 1, 1, 8, 1, [1]),
    (3, 1, 2, 2, 64, 16, [0, 1, 17]),
    (4, 1, 2, 4, 128, 16, [5, 64, 65, 700]),
    (2, 1, 1, 8, 128, 24, [1023, 129]),
    (2, 1, 1, 64, 64, 8, [300, 33]),
    (3, 7, 2, 4, 128, 16, [7, 3, 131]),
    (2, 7, 1, 2, 72, 5, [200, 64]),
    (2, 32, 1, 3, 96, 7, [500, 31]),
    (2, 17, 1, 8, 128, 64, [257, 16]),
    (2, 1, 3, 5, 256, 16, [321, 2]),
    (1, 5, 2, 8, 256, 16, [77]),
    (5, 2, 1, 1, 80, 3, [1, 2, 3, 64, 190]),
    (70, 1, 1, 2, 64, 16, [(37 * i) % 150 for i in range(70)]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Q,H,G,D,page,lengths", CASES)
def test_matches_the_oracle(dtype, B, Q, H, G, D, page, lengths):
    args = _make(B, Q, H, G, D, page, lengths, dtype, 11 + Q + D, head_major=B % 2 == 0, fill=float("nan"))
    _check(*args)
    assert P.check() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (63, 4), (64, 64), (65, 100), (500, 3), (1000, 5), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows_and_sinks(dtype, window, sinks):
    for Q in (1, 6):
        args = _make(5, Q, 2, 3, 64, 16, [0, 3, 64, 301, 620], dtype, window % 97 + Q)
        _check(*args, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_queries_of_different_numbers(dtype):
    args = _make(6, 5, 2, 2, 64, 8, [0, 4, 5, 100, 130, 70], dtype, 5)
    n = torch.tensor([2, 5, 0, 1, 5, 3], dtype=torch.int32, device=DEV)
    _check(*args, n_query=n)
    _check(*args, n_query=n, window=20, sinks=2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("strange", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_seen_has_no_influence(dtype, strange):
    """Keys and values that are not finite, at positions that some queries see and others do not, and in slots that hold none."""
    Q = 5
    q, k, v, table, length = _make(3, Q, 1, 3, 64, 8, [4, 90, 300], dtype, 9, fill=strange)
    for b, n in enumerate(length.tolist()):
        for x in (n - 1, n - 2):
            page_id = int(table[b, x // 8])
            v[page_id, x % 8] = strange
    k[int(table[1, 89 // 8]), 89 % 8] = strange
    out, lse, st = P.paged_attention(q, k, v, table, length)
    # queries in front of the last two positions see none of it
    want, wl, _ = O.paged_attention(_np(q), np.nan_to_num(_np(k)), np.nan_to_num(_np(v)), table.cpu().numpy(), length.cpu().numpy(), 0.125)
    o = _np(out)
    for j in range(Q - 2):
        assert np.all(np.isfinite(o[:, j])) and np.abs(o[:, j] - want[:, j]).max() < 0.05
    assert not np.isfinite(o[1, Q - 1]).any() and not np.isfinite(o[2, Q - 1]).any()
    # ... and a window's queries none of what lies in front of it
    q, k, v, table, length = _make(2, Q, 1, 3, 64, 8, [200, 300], dtype, 10)
    for b, n in enumerate(length.tolist()):
        for x in range(2, n - 20 - Q + 1):
            v[int(table[b, x // 8]), x % 8] = strange
            k[int(table[b, x // 8]), x % 8] = strange
    x = 200 - 20 - Q + 1                                   # seen by the first query alone
    v[int(table[0, x // 8]), x % 8] = strange
    out, lse, st = P.paged_attention(q, k, v, table, length, window=20, sinks=2)
    o = _np(out)
    assert not np.isfinite(o[0, 0]).any() and np.isfinite(o[0, 1:]).all() and np.isfinite(o[1]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_flagged_sequences(dtype):
    q, k, v, table, length = _make(6, 2, 2, 2, 64, 16, [40, 300, 50, 60, 200, 64], dtype, 21)
    length[0], length[1] = -1, table.shape[1] * 16 + 1
    table[2, 1], table[3, 3] = k.shape[0], -5               # the last page of sequences 2 and 3
    table[4, 0] = 1 << 30
    P.check()
    got = _check(q, k, v, table, length)
    assert got[2].tolist() == [256, 256, 128, 128, 128, 0]
    assert P.check() == 5
    got = _check(q, k, v, table, length, window=30)        # sequence 4 does not see its bad page then
    assert got[2].tolist() == [256, 256, 128, 128, 0, 0]
    got = _check(q, k, v, table, length, n_query=torch.tensor([1, 1, 0, 3, -1, 2], dtype=torch.int32, device=DEV))
    assert got[2].tolist() == [256, 256, 0, 256, 256, 0]
    P.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_bad_page_in_a_piece_of_a_long_sequence(dtype):
    q, k, v, table, length = _make(2, 1, 1, 2, 64, 16, [20000, 3000], dtype, 22)
    table[0, 700] = -1
    out, lse, st = P.paged_attention(q, k, v, table, length)
    assert st.tolist() == [128, 0] and float(out[0].abs().max()) == 0 and torch.isneginf(lse[0]).all() and float(out[1].abs().min()) > 0
    P.check()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_orders(dtype):
    """q and out as views, tables wider than they need be, q anywhere in memory; scale given."""
    q, k, v, table, length = _make(3, 4, 2, 2, 64, 16, [10, 100, 150], dtype, 31)
    wide = torch.randn((4, 3, 4, 130), device=DEV).to(dtype)
    qv = wide.permute(1, 0, 2, 3)[..., 1:65]               # [B, Q, Hq, D], odd start, positions outermost
    out = torch.full((3, 4, 4, 67), 7.0, dtype=dtype, device=DEV)
    got = _check(qv, k, v, table, length, scale=0.3, out=out[..., 3:])
    assert got[0].data_ptr() == out[..., 3:].data_ptr() and float((out[..., :3] - 7).abs().max()) == 0
    both = torch.stack([k, v], 2)                          # keys and values side by side in one pool
    _check(q, both[:, :, 0], both[:, :, 1], torch.cat([table, table], 1)[:, :table.shape[1]], length, scale=-0.2)
    _check(q, k, v, table, length, scale=0.0)


@pytest.mark.parametrize("dtype,G,Q,D", [(BF16, 4, 1, 128), (BF16, 4, 7, 128), (BF16, 8, 8, 64), (F32, 2, 1, 128), (F32, 3, 3, 80)])
def test_long_and_ragged(dtype, G, Q, D):
    """Sequences that are cut in many pieces, beside short ones; against float64 on the GPU."""
    lengths = [33000, 1, 5, 9000, 64, 128, 20001, 0]
    q, k, v, table, length = _make(8, Q, 2, G, D, 16, lengths, dtype, 41 + Q)
    out, lse, st = P.paged_attention(q, k, v, table, length)
    for b, n in enumerate(lengths):
        if n < Q:
            continue
        ids = table[b, :-(-n // 16)].long()
        kk, vv = (t[ids].reshape(-1, 2, D)[:n].double() for t in (k, v))
        for j in range(Q):
            p = n - Q + j
            w = torch.einsum("hgd,xhd->hgx", q[b, j].double().view(2, G, D), kk[:p + 1]) / D ** 0.5
            want = torch.einsum("hgx,xhd->hgd", torch.softmax(w, -1), vv[:p + 1]).reshape(2 * G, D)
            size = torch.einsum("hgx,xhd->hgd", torch.softmax(w, -1), vv[:p + 1].abs()).reshape(2 * G, D)
            e = (D + 4) * 2.0 ** -23 * float(q[b, j].double().norm(dim=-1).max() * kk.norm(dim=-1).max()) / D ** 0.5
            # (sums over n positions are joined from tiles and pieces of them: far fewer than n roundings follow one another)
            share = 2 * (e + 2.0 ** -21 + (2.0 ** -16 if dtype == BF16 else 0) + 2048 * 2.0 ** -23)
            err = (out[b, j].double() - want).abs()
            assert bool((err <= torch.finfo(dtype).eps / 2 * 1.01 * want.abs() + share * size).all()), (b, j, float(err.max()))
            ll = torch.logsumexp(w, -1).reshape(-1)
            assert float((lse[b, j].double() - ll).abs().max()) <= e + 2.0 ** -21 + 2048 * 2.0 ** -23 + 2.0 ** -22 * float(ll.abs().max())
    assert float(out[7].abs().max()) == 0 and torch.isneginf(lse[7]).all()
    again = P.paged_attention(q, k, v, table, length)
    assert all(torch.equal(a, b) for a, b in zip((out, lse, st), again))


def test_offsets_beyond_32_bits():
    n_pages, page, H, D = 70000, 16, 8, 256                # 4.6 GB a pool
    k = torch.zeros((n_pages, page, H, D), dtype=BF16, device=DEV)
    q, ks, vs, table, length = _make(1, 1, H, 2, D, page, [50], BF16, 51)
    far = [n_pages - 1 - i for i in range(4)]
    k[far] = ks[table[0, :4].long()]
    t = torch.tensor([far], dtype=torch.int32, device=DEV)
    out, lse, _ = P.paged_attention(q, k, k, t, length)
    want, wl, _ = P.paged_attention(q, ks, ks, table, length)
    assert torch.equal(out, want) and torch.equal(lse, wl)


def test_captured_calls_and_other_streams():
    q, k, v, table, length = _make(4, 1, 2, 4, 128, 16, [3000, 10, 500, 64], BF16, 61)
    want = P.paged_attention(q, k, v, table, length)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = P.paged_attention(q, k, v, table, length, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, P.paged_attention(q, k, v, table, length)))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        for st, (graph, _) in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for _, o in graphs:
        assert all(torch.equal(a, b) for a, b in zip(o, want))
    length[1] = 170                                        # lengths are read when the graph runs
    table[1, :11] = table[0, :11]
    graphs[0][0].replay()
    torch.cuda.synchronize()
    _check(q, k, v, table, length, got=graphs[0][1])


def test_the_binding_refuses():
    q, k, v, table, length = _make(2, 2, 2, 2, 64, 16, [20, 30], BF16, 71)
    call = P.paged_attention
    for bad in (lambda: call(q[0], k, v, table, length), lambda: call(q, k[..., :32], v, table, length), lambda: call(q, k, v[1:], table, length),
                lambda: call(q, k.float(), v, table, length), lambda: call(q, k, v, table[:1], length), lambda: call(q, k, v, table.long(), length),
                lambda: call(q, k, v, table, length.long()), lambda: call(q, k, v, table, length[:1]), lambda: call(q, k, v, table.cpu(), length),
                lambda: call(q, k, v, table, length, window=-1), lambda: call(q, k, v, table, length, out=q.float()),
                lambda: call(q.half(), k.half(), v.half(), table, length), lambda: call(q.transpose(2, 3).contiguous().transpose(2, 3), k, v, table, length),
                lambda: call(q, k, v, table, length, n_query=length[:1])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call(q[:, :, :3], k, v, table, length), lambda: call(q, k, v, table, length, scale=float("inf")),
                lambda: call(q[..., :4], k[..., :4], v[..., :4], table, length), lambda: call(q[:, :0], k, v, table, length),
                lambda: call(q.repeat(1, 17, 1, 1), k, v, table, length), lambda: call(q[..., :8], k[..., 1:9], v[..., :8], table, length)):
        with pytest.raises(P.SakiError):
            bad()
