"""Beam searches whose logits come from attention over the cache that the beams share: which beam and token every choice is, step by step.

A choice is checked by itself: its key, in float64 from the logits that the call was given, is the score it reports (to the 4e-6 and the rounding of
test_gpu_beam_select), no pair of beam and token is chosen twice in a group, and where the oracle's keys around a choice are further apart than twice that, it is the oracle's."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2609_36601_b200 as P
from test_gpu_beam_select import LSE
from test_gpu_rollout_runs import BF16, DEV, _holds, _Model, _pools

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _nothing_flagged():
    """The count of flagged rows is the library's: what other tests left in it goes first."""
    P.check()


def _choices(out, logits, score, finished, pad):
    """Returns how many choices the oracle decided."""
    B, W, V = logits.shape
    n = out["token"].shape[1]
    z, s, f = logits.double().cpu().numpy(), score.double().cpu().numpy(), finished.cpu().numpy()
    keys = np.full((B, W, V), -np.inf)
    for b in range(B):
        for w in range(W):
            if s[b, w] == -np.inf:
                continue
            if f[b, w]:
                keys[b, w, pad] = s[b, w]
            else:
                m = z[b, w].max()
                keys[b, w] = s[b, w] + (z[b, w] - m - np.log(np.exp(z[b, w] - m).sum()))
    parent, token, best, _ = O.beam_select(z, s, n, 1.0, f, pad)
    wide = O.beam_select(z, s, n + 1, 1.0, f, pad)[2]
    p, t, got = (out[k].cpu().numpy() for k in ("parent", "token", "score"))
    decided = 0
    for b in range(B):
        assert len({(x, y) for x, y in zip(p[b], t[b])}) == n
        for i in range(n):
            key = keys[b, p[b, i], t[b, i]]
            assert np.isfinite(key) and abs(got[b, i] - key) <= LSE + 2.0 ** -24 * abs(key), (b, i)
            apart = min([wide[b, i - 1] - wide[b, i]] * (i > 0) + [wide[b, i] - wide[b, i + 1]])
            if apart > 2 * LSE:
                assert (p[b, i], t[b, i]) == (parent[b, i], token[b, i]), (b, i)
                decided += 1
    return decided


@pytest.mark.parametrize("dtype,page,D,W", [(BF16, 16, 128, 4), (BF16, 8, 64, 7), (torch.float32, 5, 24, 3)])
def test_every_choice_of_a_search(dtype, page, D, W):
    B, V, steps, prompt = 3, 300, 25, 9
    m = _Model(V, 2, 2, D, 1, dtype, 17)
    rows = B * W
    cache = P.PageCache.empty(rows, 48 // page + 2, rows * (48 // page + 2), page, DEV)
    pools = _pools(m, cache.n_pages, page)
    rng = np.random.default_rng(2)
    first = torch.tensor(rng.integers(1, V, (B, prompt)), device=DEV).repeat_interleave(W, 0)
    n_new = torch.tensor([prompt if w == 0 else 0 for _ in range(B) for w in range(W)], dtype=torch.int32, device=DEV)
    _, _, st = P.cache_reserve(cache, n_new)
    P.cache_write(cache, *m.kv(0, first, torch.zeros(rows, dtype=torch.int64, device=DEV)), *pools, st, n_new)
    P.cache_fork(cache, torch.zeros(rows, dtype=torch.int32, device=DEV), W)
    history = [r.tolist() for r in first]
    score = torch.tensor([[0.0] + [-float("inf")] * (W - 1)] * B, device=DEV)
    finished = torch.zeros((B, W), dtype=torch.uint8, device=DEV)
    token, decided = first[:, -1:], 0
    for step in range(steps):
        if step:
            at = cache.length.long()
            src, dst, st = P.cache_reserve(cache, 1)
            P.copy_pages(pools, src, dst)
            P.cache_write(cache, *m.kv(0, token, at), *pools, st)
            for h, x in zip(history, token[:, 0].tolist()):
                h.append(x)
        out, _, _ = P.paged_attention(m.queries(token, cache.length.long() - 1), *pools, cache.page_table, cache.length, row_status=st if step else None)
        logits = (out.float().flatten(1) @ m.head.T).view(B, W, V).to(dtype)
        best = P.beam_select(logits, score, W, finished=finished, pad=0)
        decided += _choices(best, logits, score, finished, 0)
        p = best["parent"]
        assert int(P.cache_fork(cache, p.flatten().contiguous(), W).abs().max()) == 0
        history = [list(history[b * W + int(p[b, w])]) for b in range(B) for w in range(W)]
        finished = torch.gather(finished, 1, p.long()) | (best["token"] == 5).to(torch.uint8)
        score, token = best["score"], best["token"].flatten()[:, None].long()
    _holds(m, cache, pools, history)
    assert decided > steps * B * W // 2
    assert P.check() == 0
