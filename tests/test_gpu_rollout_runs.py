"""The cache, attention, beam selection and block verification together, as a decoder uses them, against what the histories of the sequences say.

Keys and values here are functions of a token and its position, so the cache of a sequence can be told from its tokens alone: the pages
hold copies (equal to the bit), attention is compared with float64 over the history (tolerances: those of test_gpu_paged_attention, at its _check)."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P
from test_gpu_paged_attention import _check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


class _Model:
    """Tables that keys, values, queries and logits come from."""

    def __init__(self, V, H, G, D, layers, dtype, seed, longest=400):
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)
        self.V, self.H, self.G, self.D, self.layers, self.dtype = V, H, G, D, layers, dtype
        self.k, self.v = r(layers, V, H, D), r(layers, V, H, D)
        self.q, self.at, self.head = r(V, H * G, D), r(longest, 1, D), r(V, H * G * D) / 8

    def kv(self, layer, tokens, first):                        # tokens [B, Q], first [B]: position of the first
        p = (first[:, None] + torch.arange(tokens.shape[1], device=DEV)).clamp(min=0)
        return [(t[layer][tokens] + self.at[p]).to(self.dtype) for t in (self.k, self.v)]

    def queries(self, tokens, first):
        p = (first[:, None] + torch.arange(tokens.shape[1], device=DEV)).clamp(min=0)
        return (self.q[tokens] + self.at[p]).to(self.dtype)


def _pools(m, n_pages, page):
    return [torch.full((n_pages, page, m.H, m.D), float("nan"), dtype=m.dtype, device=DEV) for _ in range(2 * m.layers)]


def _holds(m, cache, pools, history):
    """The pages of every sequence hold its history, no page is shared that should not be, and counts say who holds what."""
    assert cache.length.tolist() == [len(h) for h in history]
    counts = [0] * cache.n_pages
    for b, h in enumerate(history):
        n = len(h)
        ids = cache.page_table[b].tolist()
        for i in ids[:-(-n // cache.page_size)]:
            counts[i] += 1
        if n:
            page = cache.page_table[b, :-(-n // cache.page_size)].long()
            tokens = torch.tensor([h], device=DEV)
            for layer in range(m.layers):
                for pool, want in zip(pools[2 * layer:], m.kv(layer, tokens, torch.zeros(1, dtype=torch.int64, device=DEV))):
                    assert torch.equal(pool[page].flatten(0, 1)[:n], want[0])
    assert cache.ref_count.tolist() == counts


@pytest.mark.parametrize("dtype,page,D", [(BF16, 8, 64), (BF16, 16, 128), (torch.float32, 5, 24)])
def test_a_beam_search(dtype, page, D):
    B, W, V, steps = 3, 4, 300, 30
    m = _Model(V, 2, 2, D, 2, dtype, 7)
    prompts = [3, 16, 21]
    rows = B * W
    cache = P.PageCache.empty(rows, 64 // page + 2, rows * (64 // page + 2), page, DEV)
    pools = _pools(m, cache.n_pages, page)
    rng = np.random.default_rng(1)
    history = [rng.integers(1, V, n).tolist() for n in prompts for _ in range(1)]
    # the prompt goes into the first beam of a group, the others take its pages
    longest = max(prompts)
    n_new = torch.tensor([prompts[b] if w == 0 else 0 for b in range(B) for w in range(W)], dtype=torch.int32, device=DEV)
    tokens = torch.zeros((rows, longest), dtype=torch.int64, device=DEV)
    for b, h in enumerate(history):
        tokens[b * W, longest - len(h):] = torch.tensor(h, device=DEV)
    src, dst, st = P.cache_reserve(cache, n_new)
    assert int(st.abs().max()) == 0 and int(src.max()) == -1
    for layer in range(m.layers):
        # row j < n_new of the call is position length - n_new + j: the rows that are used come first
        t = torch.zeros_like(tokens)
        for b, h in enumerate(history):
            t[b * W, :len(h)] = torch.tensor(h, device=DEV)
        k, v = m.kv(layer, t, torch.zeros(rows, dtype=torch.int64, device=DEV))
        P.cache_write(cache, k, v, pools[2 * layer], pools[2 * layer + 1], st, n_new)
    assert int(P.cache_fork(cache, torch.zeros(rows, dtype=torch.int32, device=DEV), W).abs().max()) == 0
    history = [list(history[b]) for b in range(B) for _ in range(W)]
    _holds(m, cache, pools, history)
    score = torch.tensor([[0.0] + [-float("inf")] * (W - 1)] * B, device=DEV)
    finished = torch.zeros((B, W), dtype=torch.uint8, device=DEV)
    token = torch.tensor([[h[-1]] for h in history], device=DEV)
    copies = 0
    for step in range(steps):
        if step:                                               # the chosen tokens' keys and values
            first = cache.length.long()
            src, dst, st = P.cache_reserve(cache, 1)
            assert int(st.abs().max()) == 0
            copies += int((src >= 0).sum())
            P.copy_pages(pools, src, dst)
            for layer in range(m.layers):
                P.cache_write(cache, *m.kv(layer, token, first), pools[2 * layer], pools[2 * layer + 1], st)
            for h, t in zip(history, token[:, 0].tolist()):
                h.append(t)
        last = cache.length.long() - 1
        hidden = []
        for layer in range(m.layers):
            args = (m.queries(token, last), pools[2 * layer], pools[2 * layer + 1], cache.page_table, cache.length)
            got = P.paged_attention(*args)
            if step % 7 == 0:
                _check(*args, got=got)
            hidden.append(got[0].float().flatten(1))
        logits = ((hidden[0] + hidden[1]) @ m.head.T).view(B, W, V).to(dtype)
        # beams that are alike in all but their scores have equal keys nowhere: the oracle decides where keys are apart
        out = P.beam_select(logits, score, W, finished=finished, pad=0)
        parent, tok, best, _ = O.beam_select(logits.double().cpu().numpy(), score.double().cpu().numpy(), W, 1.0, finished.cpu().numpy(), 0)
        assert np.allclose(out["score"].cpu().numpy(), best, rtol=2.0 ** -23, atol=4e-6)
        p = out["parent"]
        assert int(P.cache_fork(cache, p.flatten().contiguous(), W).abs().max()) == 0
        history = [list(history[b * W + int(p[b, w])]) for b in range(B) for w in range(W)]
        finished = torch.gather(finished, 1, p.long()) | (out["token"] == 5).to(torch.uint8)
        score, token = out["score"], out["token"].flatten()[:, None].long()
        if step % 5 == 0:
            _holds(m, cache, pools, history)
    assert copies > 0
    src, dst, moves = P.cache_compact(cache)
    P.copy_pages(pools, src, dst)
    _holds(m, cache, pools, history)
    used = int((cache.ref_count > 0).sum())
    assert int((cache.ref_count[:used] > 0).sum()) == used
    P.check()


@pytest.mark.parametrize("captured", [False, True])
def test_verified_blocks(captured):
    """Drafted blocks: reserve, write, attend, verify, cut back to what was accepted; eager, and as one captured step that is replayed."""
    B, K, V, page = 5, 4, 400, 8
    m = _Model(V, 2, 3, 64, 1, BF16, 11)
    cache = P.PageCache.empty(B, 40, 120, page, DEV)
    pools = _pools(m, cache.n_pages, page)
    rng = np.random.default_rng(3)
    history = [rng.integers(0, V, n).tolist() for n in (1, 7, 8, 9, 30)]
    n_new = torch.tensor([len(h) for h in history], dtype=torch.int32, device=DEV)
    t = torch.zeros((B, 30), dtype=torch.int64, device=DEV)
    for b, h in enumerate(history):
        t[b, :len(h)] = torch.tensor(h, device=DEV)
    _, _, st = P.cache_reserve(cache, n_new)
    P.cache_write(cache, *m.kv(0, t, torch.zeros(B, dtype=torch.int64, device=DEV)), *pools, st, n_new)
    block = torch.zeros((B, K + 1), dtype=torch.int64, device=DEV)       # the token after the cache's last, then the drafted ones
    s = torch.zeros((B, K + 1, V), dtype=BF16, device=DEV)

    def step():
        first = cache.length.long()
        src, dst, st = P.cache_reserve(cache, K + 1)
        P.copy_pages(pools, src, dst)
        P.cache_write(cache, *m.kv(0, block, first), *pools, st)
        args = (m.queries(block, first), *pools, cache.page_table, cache.length)
        got = P.paged_attention(*args)
        logits = (got[0].float().flatten(2) @ m.head.T).to(BF16)
        verdict = P.spec_verify(s, logits, block[:, 1:].int().contiguous(), 0.2, seed=5)
        lengths = cache.length.clone()
        kept = P.cache_truncate(cache, verdict["n_accept"], of=K + 1, keep_add=1)
        return st, args, got, verdict, kept, lengths

    def fill(i):
        g = torch.Generator(device=DEV).manual_seed(100 + i)
        block.copy_(torch.randint(0, V, (B, K + 1), generator=g, device=DEV))
        s.copy_((2 * torch.randn((B, K + 1, V), generator=g, device=DEV)).to(BF16))

    graph = None
    if captured:
        before, kept_pools = cache.meta.clone(), [p.clone() for p in pools]
        fill(0)
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = step()
        cache.meta.copy_(before)
        for p, w in zip(pools, kept_pools):
            p.copy_(w)
    accepted = 0
    for i in range(12):
        fill(i)
        if captured:
            graph.replay()
            st, args, got, verdict, kept, lengths = result
        else:
            st, args, got, verdict, kept, lengths = step()
        assert int(st.abs().max()) == 0 and int(kept.abs().max()) == 0
        n = verdict["n_accept"].tolist()
        accepted += sum(n)
        if not captured:                                       # (the tables now are those after the cut: a longer one than was kept is gone)
            whole = [h + block[b].tolist() for b, h in enumerate(history)]
            for b, h in enumerate(whole):
                assert int(lengths[b]) == len(h)
        history = [h + block[b, :n[b] + 1].tolist() for b, h in enumerate(history)]
        _holds(m, cache, pools, history)
        # queries of what was kept see only what was kept: compare those with a call on the cache as it is now
        nq = (verdict["n_accept"] + 1).int()
        again = P.paged_attention(m.queries(block, cache.length.long() - nq.long()), *pools, cache.page_table, cache.length, n_query=nq)
        q = m.queries(block, cache.length.long() - nq.long())
        _check(q, *pools, cache.page_table, cache.length, n_query=nq, got=again)
        for b in range(B):                                     # (tiles start elsewhere in the two calls for nothing: positions are the same)
            c = int(nq[b])
            assert torch.equal(got[1][b, :c], again[1][b, :c]) or torch.allclose(got[1][b, :c], again[1][b, :c], rtol=0, atol=1e-5)
    assert accepted > 0
    assert P.check() == 0
