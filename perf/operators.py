"""Operators around the routing of a rollout, measured: attention over a paged key-value cache, the pages of such a cache, and
beam selection over vocabulary rows, at the sizes that a program around this library meets.

A case names an operator (`op`):

  attention  paged_attention: new tokens (one, or a drafted block) over a paged cache
  block      cache_reserve, cache_write, cache_truncate: a drafted block goes into the cache, its accepted prefix stays
  fork       cache_fork, cache_reserve, copy_pages: the cache follows the parents that beam selection chose
  compact    cache_compact, copy_pages: the used pages move to the front of the pool
  beams      beam_select: the best continuations of every group of beams

`own` false: the plain forms, elementary torch operations.  `own` true: the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NEG = -math.inf


def listed():
    return [
        # the first tokens of one rollout: a single sequence, one new token; launches and latency count
        dict(name="attn_one", op="attention", B=1, Q=1, H=8, G=2, D=128, page=16, lo=1000, hi=1000, dtype="bf16", window=0, sinks=0, head_major=False),
        # a serving batch of sequences at all stages of their generation
        dict(name="attn_batch", op="attention", B=64, Q=1, H=8, G=4, D=128, page=16, lo=1, hi=8191, dtype="bf16", window=0, sinks=0, head_major=False),
        # verification of drafted blocks: 512 sequences, six drafted tokens and the one before them
        dict(name="attn_verify", op="attention", B=512, Q=7, H=8, G=4, D=128, page=16, lo=65, hi=2048, dtype="bf16", window=0, sinks=0, head_major=False),
        # one long context, many query heads on few key heads, pages as large as they get
        dict(name="attn_long", op="attention", B=1, Q=1, H=4, G=8, D=128, page=64, lo=131077, hi=131077, dtype="bf16", window=0, sinks=0, head_major=True),
        # a layer with a sliding window and four first tokens that stay visible, heads of 64
        dict(name="attn_window", op="attention", B=96, Q=1, H=8, G=5, D=64, page=32, lo=700, hi=16000, dtype="bf16", window=1024, sinks=4, head_major=True),
        # a cache kept in fp32 (small batch, odd heads and pages)
        dict(name="attn_f32", op="attention", B=24, Q=3, H=3, G=3, D=80, page=24, lo=5, hi=3001, dtype="f32", window=0, sinks=0, head_major=False),
        # a drafted block of a small batch goes into one layer's cache
        dict(name="block_8", op="block", B=8, Q=7, H=8, D=128, page=16, lo=100, hi=2000, dtype="bf16", n_pages=2048),
        # ... and of 512 sequences
        dict(name="block_512", op="block", B=512, Q=7, H=8, D=128, page=16, lo=65, hi=1900, dtype="bf16", n_pages=40000),
        # 64 groups of 8 beams take their parents' pages; four layers' keys and values are copied where pages part
        dict(name="fork_64x8", op="fork", groups=64, W=8, H=8, D=128, page=16, lo=60, hi=1000, dtype="bf16", layers=4),
        # a half empty pool is moved together, two layers
        dict(name="compact_8192", op="compact", B=128, H=8, D=128, page=16, n_pages=8192, used=4096, dtype="bf16", layers=2),
        # beam search of one prompt
        dict(name="beams_1x4", op="beams", B=1, W=4, n=4, V=151936, dtype="bf16", temperature=1.0, finished=False),
        # a batch of prompts with eight beams each, some of them finished
        dict(name="beams_64x8", op="beams", B=64, W=8, n=8, V=151936, dtype="bf16", temperature=1.0, finished=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "block", "fork", "compact", "beams", "beams"))
    if op == "attention":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        H, G = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 3, 4, 5, 8))
        D = rng.choice((64, 72, 80, 96, 128, 128, 256)) if dtype == "bf16" else rng.choice((36, 64, 80, 128))
        Q = rng.choice((1, 1, rng.randint(2, 17)))
        # positions of all sequences together, at most half of those of the largest listed cache
        total = _log_int(rng, 300, int(2.5e8 / (H * D * (2 if dtype == "f32" else 1)) / max(1, Q * G // 32)))
        B = min(512, _log_int(rng, 1, max(2, total // 64)))
        hi = max(2, min(140000, 2 * total // B))
        lo = hi if B == 1 else rng.randint(1, hi)
        window = rng.choice((0, 0, 0, _log_int(rng, 16, 4096)))
        return dict(op=op, B=B, Q=Q, H=H, G=G, D=D, page=rng.choice((8, 16, 16, 24, 32, 64)), lo=lo, hi=hi, dtype=dtype, window=window,
                    sinks=rng.choice((0, 1, 4, 20)) if window else 0, head_major=rng.random() < 0.5)
    if op == "block":
        B, page = _log_int(rng, 1, 512), rng.choice((8, 16, 24, 64))
        hi = _log_int(rng, 40, 2000)
        return dict(op=op, B=B, Q=rng.choice((1, rng.randint(2, 17))), H=rng.choice((1, 2, 4, 8)), D=rng.choice((64, 80, 128)), page=page,
                    lo=rng.randint(1, hi), hi=hi, dtype=rng.choice(("bf16", "bf16", "f32")), n_pages=B * (hi // page + 4) + rng.randint(0, 3000))
    if op == "fork":
        groups, W = _log_int(rng, 1, 64), rng.choice((2, 3, 4, 5, 8))
        hi = _log_int(rng, 20, 1000)
        return dict(op=op, groups=groups, W=W, H=rng.choice((1, 2, 4, 8)), D=rng.choice((64, 80, 128)), page=rng.choice((8, 16, 24)),
                    lo=rng.randint(1, hi), hi=hi, dtype=rng.choice(("bf16", "bf16", "f32")), layers=rng.randint(1, 4))
    if op == "compact":
        n_pages = _log_int(rng, 200, 8192)
        return dict(op=op, B=_log_int(rng, 4, 128), H=rng.choice((1, 2, 4, 8)), D=rng.choice((64, 80, 128)), page=rng.choice((8, 16)),
                    n_pages=n_pages, used=rng.randint(150, n_pages - 10), dtype="bf16", layers=rng.randint(1, 2))
    W, dtype = rng.randint(2, 12), rng.choice(("bf16", "bf16", "f32"))
    V = _log_int(rng, 1000, 160000)
    return dict(op=op, B=min(64, _log_int(rng, 1, max(2, int((7e7 if dtype == "bf16" else 3.5e7) / V / W)))), W=W, n=rng.choice((W, W, min(32, 2 * W))), V=V, dtype=dtype,
                temperature=rng.choice((1.0, 1.0, 0.75, 1.25)), finished=rng.random() < 0.5)


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * 7 + seed)


def _type(case):
    return BF16 if case["dtype"] == "bf16" else F32


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lengths(case, n):
    """n lengths from lo to hi, evenly spaced: the same set for every seed."""
    lo, hi = case["lo"], case["hi"]
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device=DEV, dtype=dtype)


def _pools(case, gen, n_pages, n, head_major=False):
    shape = (n_pages, case["H"], case["page"], case["D"]) if head_major else (n_pages, case["page"], case["H"], case["D"])
    pools = [_randn(gen, shape, _type(case)) for _ in range(n)]
    return [p.transpose(1, 2) for p in pools] if head_major else pools


def _tables(counts, max_pages, ids):
    """Page tables: counts[b] of the page ids each, in order, and -1 behind them."""
    at = torch.arange(max_pages, device=DEV)[None, :]
    start = torch.cumsum(counts, 0) - counts
    have = at < counts[:, None]
    return torch.where(have, ids[(start[:, None] + at).clamp(max=max(0, ids.numel() - 1))], -1).to(torch.int32)


def _meta(table, length, ref):
    """A cache's tables in one tensor, as a program keeps them: page table, lengths, counts of holders."""
    return torch.cat([table.reshape(-1), length, ref]).to(torch.int32)


def _shuffled(values, gen):
    v = torch.tensor(values, device=DEV, dtype=torch.int32)
    return v[torch.randperm(v.numel(), generator=gen, device=DEV)]


def prepare(case, seed):
    gen, op = _gen(seed), case["op"]
    s = dict(case=case)
    if op == "attention":
        B, Q, H, G, D, page = (case[k] for k in ("B", "Q", "H", "G", "D", "page"))
        length = _shuffled(_lengths(case, B), gen)
        counts = (length + page - 1) // page
        max_pages = (case["hi"] + page - 1) // page
        n_pages = sum((x + page - 1) // page for x in _lengths(case, B)) + 7
        ids = torch.randperm(n_pages, generator=gen, device=DEV)
        s["k"], s["v"] = _pools(case, gen, n_pages, 2, case["head_major"])
        s["q"] = (2 * _randn(gen, (B, Q, H * G, D), F32)).to(_type(case))
        s["table"], s["length"] = _tables(counts, max_pages, ids), length
        return s
    if op == "block":
        B, Q, page, n_pages = (case[k] for k in ("B", "Q", "page", "n_pages"))
        length = _shuffled(_lengths(case, B), gen)
        counts = (length + page - 1) // page
        max_pages = (case["hi"] + Q + page - 1) // page
        ids = torch.randperm(n_pages, generator=gen, device=DEV)
        table = _tables(counts, max_pages, ids)
        ref = torch.zeros(n_pages + 1, device=DEV, dtype=torch.int32)
        ref[table.long().reshape(-1)] = 1             # (the entries -1 mark the last, which is cut off)
        s["meta"], s["sizes"] = _meta(table, length, ref[:n_pages]), (B, max_pages, n_pages, page)
        s["k"], s["v"] = _pools(case, gen, n_pages, 2)
        shape = (B, Q, case["H"], case["D"])
        s["new_k"], s["new_v"] = _randn(gen, shape, _type(case)), _randn(gen, shape, _type(case))
        s["keep"] = torch.randint(0, Q + 1, (B,), generator=gen, device=DEV, dtype=torch.int32)
        return s
    if op == "fork":
        groups, W, page = case["groups"], case["W"], case["page"]
        B = groups * W
        glen = _shuffled(_lengths(case, groups), gen)
        gcount = (glen + page - 1) // page
        own_pages = torch.clamp(gcount, max=2)          # the last pages of a beam are its own, the ones before are its group's
        max_pages = (case["hi"] + 1 + page - 1) // page
        lens = _lengths(case, groups)
        n_shared = sum(max(0, (x + page - 1) // page - 2) for x in lens)
        n_own = W * sum(min(2, (x + page - 1) // page) for x in lens)
        n_pages = n_shared + n_own + 2 * B + 5
        ids = torch.randperm(n_pages, generator=gen, device=DEV)
        g = torch.arange(B, device=DEV) // W
        at = torch.arange(max_pages, device=DEV)[None, :]
        shared = (gcount - own_pages)[g]
        sstart = (torch.cumsum(gcount - own_pages, 0) - (gcount - own_pages))[g]
        ostart = n_shared + torch.cumsum(own_pages[g], 0) - own_pages[g]
        where = torch.where(at < shared[:, None], sstart[:, None] + at, ostart[:, None] + at - shared[:, None])
        table = torch.where(at < gcount[g][:, None], ids[where.clamp(max=n_pages - 1)], -1).to(torch.int32)
        ref = torch.bincount(table.reshape(-1).long() + 1, minlength=n_pages + 1)[1:].to(torch.int32)
        s["meta"], s["sizes"] = _meta(table, glen[g], ref), (B, max_pages, n_pages, page)
        s["pools"] = _pools(case, gen, n_pages, 2 * case["layers"])
        parents = torch.tensor(_parents(W), device=DEV, dtype=torch.int32)
        order = torch.rand((groups, W), generator=gen, device=DEV).argsort(1)
        s["parent"] = parents[order].contiguous()
        return s
    if op == "compact":
        B, n_pages, used, page = (case[k] for k in ("B", "n_pages", "used", "page"))
        counts = torch.tensor([used // B + (i < used % B) for i in range(B)], device=DEV)
        max_pages = used // B + 2
        ids = torch.randperm(n_pages, generator=gen, device=DEV)
        table = _tables(counts, max_pages, ids)
        ref = torch.zeros(n_pages + 1, device=DEV, dtype=torch.int32)
        ref[table.long().reshape(-1)] = 1
        s["meta"], s["sizes"] = _meta(table, counts * page, ref[:n_pages]), (B, max_pages, n_pages, page)
        s["pools"] = _pools(case, gen, n_pages, 2 * case["layers"])
        return s
    B, W, V = case["B"], case["W"], case["V"]
    rank = torch.argsort(torch.rand((B * W, V), generator=gen, device=DEV)) if V <= 4096 else torch.rand((B * W, V), generator=gen, device=DEV).mul_(V)
    s["logits"] = (2.0 * _randn(gen, (B * W, V), F32) - 1.1 * torch.log1p(rank.float())).to(_type(case)).view(B, W, V)
    s["score"] = -3.0 * torch.rand((B, W), generator=gen, device=DEV)
    s["finished"] = (torch.rand((B, W), generator=gen, device=DEV) < 0.25).to(torch.uint8) if case["finished"] else None
    return s


def _parents(W):
    """The parents of a group's new beams, best first: the front beams have several children, some beams none."""
    return [i * i // (2 * W) for i in range(W)]


# ---- the plain forms ----

def _plain_attention(s):
    c = s["case"]
    B, Q, H, G, D = (c[k] for k in ("B", "Q", "H", "G", "D"))
    table, length = s["table"], s["length"].long()
    pages = table.clamp(min=0).long()
    k = s["k"][pages].flatten(1, 2).float()              # [B, L, H, D]
    v = s["v"][pages].flatten(1, 2).float()
    L = k.shape[1]
    x = torch.arange(L, device=DEV)
    p = length[:, None] - Q + torch.arange(Q, device=DEV)                     # [B, Q]
    sees = x <= p[:, :, None]
    if c["window"]:
        sees &= (x > p[:, :, None] - c["window"]) | (x < c["sinks"])
    q = s["q"].float().view(B, Q, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * Q, D)
    dots = torch.matmul(q, k.permute(0, 2, 3, 1)).view(B, H, G, Q, L) * (1.0 / math.sqrt(D))
    dots = torch.where(sees[:, None, None], dots, NEG)
    m = dots.amax(-1, keepdim=True)
    e = torch.exp(dots - torch.where(m == NEG, 0.0, m))
    total = e.sum(-1, keepdim=True)
    v = torch.where((x < length[:, None])[:, :, None, None], v, 0.0).permute(0, 2, 1, 3)
    o = torch.matmul(e.view(B, H, G * Q, L), v).view(B, H, G, Q, D) / torch.where(total == 0, 1.0, total)
    lse = (m + torch.log(total)).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, Q, H * G, D).to(_type(c)), lse.permute(0, 3, 1, 2).reshape(B, Q, H * G)


def _split(s):
    B, max_pages, n_pages, page = s["sizes"]
    m = s["meta"].clone()
    return m[:B * max_pages].view(B, max_pages).long(), m[B * max_pages:B * max_pages + B].long(), m[B * max_pages + B:].long()


def _plain_reserve(table, length, ref, page, n):
    """n more positions for every sequence -> table, length, ref, pages to copy (from, to; -1: none), whether there was no room."""
    B, max_pages = table.shape
    n_pages = ref.numel()
    have, want = (length + page - 1) // page, (length + n + page - 1) // page
    last = table.gather(1, (have - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    fits = want <= max_pages
    parted = fits & (length % page != 0) & (ref[last] > 1)
    free = ref == 0
    need = torch.where(fits, want - have + parted.long(), 0)
    ok = fits & (torch.cumsum(need, 0) <= free.sum())
    writer = parted & ok
    writers = torch.zeros_like(ref).index_add(0, last, writer.long())
    at = torch.arange(B, device=table.device)
    first = torch.full_like(ref, B).scatter_reduce(0, torch.where(writer, last, 0), torch.where(writer, at, B), "amin")
    copies = writer & ~((writers == ref)[last] & (first[last] == at))
    need = torch.where(ok, want - have + copies.long(), 0)
    start = torch.cumsum(need, 0) - need
    order = torch.full((n_pages + 1,), 0, dtype=torch.long, device=table.device)
    order[torch.where(free, torch.cumsum(free, 0) - 1, n_pages)] = torch.arange(n_pages, device=table.device)
    slot = torch.arange(max_pages, device=table.device)[None, :]
    new = ok[:, None] & (slot >= have[:, None]) & (slot < want[:, None])
    own_last = copies[:, None] & (slot == have[:, None] - 1)
    rank = (start + copies.long() - have)[:, None] + slot
    rank = torch.where(own_last, start[:, None], rank).clamp(0, n_pages)
    src, dst = torch.where(copies, last, -1), torch.where(copies, order[start.clamp(max=n_pages)], -1)
    table = torch.where(new | own_last, order[rank], table)
    taken = torch.zeros(n_pages + 1, dtype=torch.long, device=table.device)
    taken[torch.where(new | own_last, table, n_pages).reshape(-1)] = 1
    ref = ref + taken[:n_pages] - torch.zeros_like(ref).index_add(0, last, copies.long())
    return table, torch.where(ok, length + n, length), ref, src, dst, ~ok


def _plain_block(s):
    c = s["case"]
    Q, page = c["Q"], c["page"]
    table, length, ref = _split(s)
    n_pages = ref.numel()
    table, length, ref, src, dst, full = _plain_reserve(table, length, ref, page, Q)
    reserved = table.to(torch.int32)
    at = length[:, None] - Q + torch.arange(Q, device=DEV)
    where = table.gather(1, at // page) * page + at % page
    for pool, new in ((s["k"], s["new_k"]), (s["v"], s["new_v"])):      # the two pools
        pool.view(n_pages * page, c["H"], c["D"])[where.reshape(-1)] = new.flatten(0, 1)
    length = length - Q + s["keep"]
    slot = torch.arange(table.shape[1], device=DEV)[None, :]
    gone = (slot >= ((length + page - 1) // page)[:, None]) & (table >= 0)
    ref = ref - torch.zeros(n_pages + 1, dtype=torch.long, device=DEV).index_add(0, torch.where(gone, table, n_pages).reshape(-1), gone.reshape(-1).long())[:n_pages]
    table = torch.where(gone, -1, table)
    i = torch.int32
    return reserved, src.to(i), dst.to(i), table.to(i), length.to(i), ref.to(i), s["k"], s["v"]


def _plain_copy(pools, src, dst):
    """Page src[i] goes to page dst[i]; where there is none, a page stays itself."""
    n = pools[0].shape[0]
    come = torch.arange(n + 1, device=src.device)
    come[torch.where(dst >= 0, dst, n)] = src
    for p in pools:
        p.copy_(p[come[:n]])


def _plain_fork(s):
    c = s["case"]
    W, page = c["W"], c["page"]
    table, length, ref = _split(s)
    B, n_pages = length.numel(), ref.numel()
    parent = (s["parent"].long() + W * torch.arange(c["groups"], device=DEV)[:, None]).reshape(-1)
    table, length = table[parent], length[parent]
    ref = torch.zeros(n_pages + 1, dtype=torch.long, device=DEV).index_add(0, torch.where(table < 0, n_pages, table).reshape(-1), torch.ones(table.numel(), dtype=torch.long, device=DEV))[:n_pages]
    table, length, ref, src, dst, full = _plain_reserve(table, length, ref, page, 1)
    _plain_copy(s["pools"], src, dst)
    i = torch.int32
    return table.to(i), length.to(i), ref.to(i), src.to(i), dst.to(i), s["pools"]


def _plain_compact(s):
    table, length, ref = _split(s)
    n_pages = ref.numel()
    ids = torch.arange(n_pages, device=DEV)
    used = ref > 0
    n_used = used.sum()
    moves, room = used & (ids >= n_used), ~used & (ids < n_used)
    half = n_pages // 2
    src, dst = (torch.full((n_pages + 1,), -1, dtype=torch.long, device=DEV) for _ in range(2))
    src[torch.where(moves, torch.cumsum(moves, 0) - 1, n_pages)] = ids
    dst[torch.where(room, torch.cumsum(room, 0) - 1, n_pages)] = ids
    src, dst = src[:half], dst[:half]
    to = torch.cat([ids, ids[:1]])
    to[torch.where(src >= 0, src, n_pages)] = torch.where(src >= 0, dst, 0)
    table = torch.where(table >= 0, to[:n_pages][table.clamp(min=0)], -1)
    count = torch.zeros_like(ref).index_add(0, to[:n_pages], ref)
    _plain_copy(s["pools"], src, dst)
    i = torch.int32
    return table.to(i), count.to(i), src.to(i), dst.to(i), moves.sum().to(i), s["pools"]


def _plain_beams(s):
    c = s["case"]
    n, V = c["n"], c["V"]
    z = s["logits"].double() / c["temperature"]
    m = z.amax(-1, keepdim=True)
    key = s["score"].double()[..., None] + (z - m - torch.log(torch.exp(z - m).sum(-1, keepdim=True)))
    if s["finished"] is not None:
        done = s["finished"].bool()
        v = torch.arange(V, device=DEV)
        key = torch.where(done[..., None], torch.where(v == 0, s["score"].double()[..., None], NEG), key)
    key = key.flatten(1)
    # the n largest, of equal ones the first: those above the n-th largest, and as many of its equals as there is room for
    bar = torch.topk(key, n).values[:, -1:]
    above, equal = key > bar, key == bar
    chosen = above | (equal & (torch.cumsum(equal, 1) <= n - above.sum(1, keepdim=True)))
    at = torch.arange(key.shape[1], device=DEV, dtype=torch.int32)
    at = -torch.topk(torch.where(chosen, -at, -2 ** 31 + 1), n).values.long()           # the chosen, lowest index first
    best, order = torch.sort(key.gather(1, at), dim=1, descending=True, stable=True)
    at = at.gather(1, order)
    none = best == NEG
    i = torch.int32
    return torch.where(none, -1, at // V).to(i), torch.where(none, -1, at % V).to(i), best.float()


# ---- the library's calls ----

def _own(s):
    import paper_2609_36601_b200 as saki
    c = s["case"]
    if c["op"] == "attention":
        out, lse, _ = saki.paged_attention(s["q"], s["k"], s["v"], s["table"], s["length"], window=c["window"], sinks=c["sinks"])
        return out, lse
    if c["op"] == "beams":
        out = saki.beam_select(s["logits"], s["score"], c["n"], temperature=c["temperature"], finished=s["finished"], pad=0)
        return out["parent"], out["token"], out["score"]
    cache = saki.PageCache(s["meta"].clone(), *s["sizes"])
    if c["op"] == "block":
        src, dst, status = saki.cache_reserve(cache, c["Q"])
        saki.cache_write(cache, s["new_k"], s["new_v"], s["k"], s["v"], status)
        reserved = cache.page_table.clone()
        saki.cache_truncate(cache, s["keep"], c["Q"])
        return reserved, src, dst, cache.page_table, cache.length, cache.ref_count, s["k"], s["v"]
    if c["op"] == "fork":
        saki.cache_fork(cache, s["parent"], c["W"])
        src, dst, status = saki.cache_reserve(cache, 1)
        saki.copy_pages(s["pools"], src, dst)
        return cache.page_table, cache.length, cache.ref_count, src, dst, s["pools"]
    src, dst, moves = saki.cache_compact(cache)
    saki.copy_pages(s["pools"], src, dst)
    return cache.page_table, cache.ref_count, src, dst, moves, s["pools"]


def run(state):
    if own:
        return _own(state)
    return {"attention": _plain_attention, "block": _plain_block, "fork": _plain_fork, "compact": _plain_compact,
            "beams": _plain_beams}[state["case"]["op"]](state)


# ---- what a pass cannot do without ----

def work(case):
    op, size = case["op"], _size(case)
    if op == "attention":
        B, Q, H, G, D = (case[k] for k in ("B", "Q", "H", "G", "D"))
        keys = pairs = 0
        for n in _lengths(case, B):
            seen = [_seen(n, n - Q + j, case["window"], case["sinks"]) for j in range(Q)]
            pairs += sum(seen)
            first = n - Q                      # the position of the first query: what any query sees
            low = max(0, first - case["window"] + 1) if case["window"] else 0
            keys += n - low + min(case["sinks"], low)
        return {"bytes": 2 * keys * H * D * size + 2 * B * Q * H * G * D * size + 4 * B * Q * H * G + 4 * keys / case["page"], "flops": 4 * pairs * H * G * D}
    if op == "block":
        B, page = case["B"], case["page"]
        tables = 4 * (B * ((case["hi"] + case["Q"]) // page + 1) + B + case["n_pages"])
        return {"bytes": 4 * B * case["Q"] * case["H"] * case["D"] * size + 2 * tables, "flops": 0}
    if op == "fork":
        B, page = case["groups"] * case["W"], case["page"]
        parted = sum(n % page != 0 for n in _lengths(case, case["groups"]))
        copies = parted * (case["W"] - len(set(_parents(case["W"]))))
        return {"bytes": 2 * copies * page * case["H"] * case["D"] * size * 2 * case["layers"] + 2 * 4 * B * (case["hi"] // page + 1), "flops": 0}
    if op == "compact":
        moves = case["used"] * (case["n_pages"] - case["used"]) // case["n_pages"]
        return {"bytes": 2 * moves * case["page"] * case["H"] * case["D"] * size * 2 * case["layers"] + 8 * case["n_pages"] + 8 * case["used"], "flops": 0}
    rows = case["B"] * case["W"]
    return {"bytes": rows * case["V"] * size + 4 * rows + 12 * case["B"] * case["n"], "flops": 3 * rows * case["V"]}


def _seen(n, p, window, sinks):
    if p < 0:
        return 0
    low = max(0, p - window + 1) if window else 0
    return p + 1 - low + min(sinks, low)


# ---- the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, s)
    if case["op"] == "beams":
        return None, None, _exact_scores(case, s)
    return None                                         # whole numbers and copies


def _exact_attention(case, s):
    B, Q, H, G, D, page = (case[k] for k in ("B", "Q", "H", "G", "D", "page"))
    out = torch.zeros((B, Q, H * G, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, Q, H * G), NEG, dtype=torch.float64, device=DEV)
    for b, n in enumerate(s["length"].tolist()):
        ids = s["table"][b, :(n + page - 1) // page].long()
        keys, values = (s[w][ids].reshape(-1, H, D)[:n].double() for w in ("k", "v"))
        for j in range(max(0, Q - n), Q):
            p = n - Q + j
            x = list(range(0, min(case["sinks"], max(0, p - case["window"] + 1)))) if case["window"] else []
            low = max(0, p - case["window"] + 1) if case["window"] else 0
            kk = torch.cat([keys[:len(x)], keys[low:p + 1]]) if x else keys[low:p + 1]
            vv = torch.cat([values[:len(x)], values[low:p + 1]]) if x else values[low:p + 1]
            q = s["q"][b, j].double().view(H, G, D)
            w = torch.bmm(q, kk.permute(1, 2, 0)) / math.sqrt(D)
            lse[b, j] = torch.logsumexp(w, -1).reshape(-1)
            out[b, j] = torch.bmm(torch.softmax(w, -1), vv.permute(1, 0, 2)).reshape(H * G, D)
    return out, lse


def _exact_scores(case, s):
    rows = []
    for b in range(case["B"]):
        logp = torch.log_softmax(s["logits"][b].double() / case["temperature"], -1) + s["score"][b].double()[:, None]
        if s["finished"] is not None:
            done = s["finished"][b].bool()
            logp[done] = NEG
            logp[done, 0] = s["score"][b].double()[done]
        rows.append(torch.sort(logp.reshape(-1), descending=True).values[:case["n"]])
    return torch.stack(rows)
