"""Float64 / integer oracle of what surrounds the routing in a rollout: the pages of a key-value cache, attention over them, and
beam selection.  One sequence, page and candidate at a time, from the definitions."""
from __future__ import annotations

import numpy as np

ST_NONFINITE, ST_BAD_ID, ST_BAD_PAGE, ST_BAD_LENGTH, ST_NO_PAGES = 8, 16, 128, 256, 512


class Cache:
    """page_table [B, max_pages], length [B], ref_count [n_pages] as Python lists."""

    def __init__(self, page_table, length, ref_count, page_size):
        self.table = [list(map(int, r)) for r in page_table]
        self.length = list(map(int, length))
        self.ref = list(map(int, ref_count))
        self.page = page_size
        self.max_pages = len(self.table[0]) if self.table else 1

    def pages(self, positions):
        return -(-positions // self.page)

    def ok(self, n):
        return 0 <= n <= self.max_pages * self.page

    def valid(self, page_id):
        return 0 <= page_id < len(self.ref)

    def reserve(self, n_new):
        B = len(self.length)
        src, dst, status = [-1] * B, [-1] * B, [0] * B
        free = [i for i, r in enumerate(self.ref) if r == 0]
        parted, counted = [False] * B, 0
        for b in range(B):
            L, n = self.length[b], n_new[b]
            if not self.ok(L) or n < 0 or not self.ok(L + n):
                status[b] = ST_BAD_LENGTH
                continue
            if n > 0 and L % self.page:
                last = self.table[b][self.pages(L) - 1]
                if not self.valid(last):
                    status[b] = ST_BAD_PAGE
                    continue
                parted[b] = self.ref[last] > 1
            counted += self.pages(L + n) - self.pages(L) + parted[b]
            if counted > len(free):
                status[b] = ST_NO_PAGES
        writers = {}
        for b in range(B):
            if parted[b] and not status[b]:
                writers.setdefault(self.table[b][self.pages(self.length[b]) - 1], []).append(b)
        keeps = {w[0] for page, w in writers.items() if len(w) == self.ref[page]}
        copies = {b for w in writers.values() for b in w if b not in keeps}
        for b in range(B):
            if status[b]:
                continue
            L, n = self.length[b], n_new[b]
            have, want = self.pages(L), self.pages(L + n)
            if b in copies:
                src[b], dst[b] = self.table[b][have - 1], free.pop(0)
                self.table[b][have - 1] = dst[b]
                self.ref[src[b]] -= 1
                self.ref[dst[b]] = 1
            for x in range(have, want):
                self.table[b][x] = free.pop(0)
                self.ref[self.table[b][x]] = 1
            self.length[b] = L + n
        return src, dst, status

    def truncate(self, keep, of=None, row_status=None):
        status = [0] * len(self.length)
        for b, k in enumerate(keep):
            if row_status is not None and row_status[b]:
                status[b] = row_status[b]
                continue
            L = self.length[b]
            last = L if of is None else of
            if not self.ok(L) or last > L or not 0 <= k <= last:
                status[b] = ST_BAD_LENGTH
                continue
            left = L - last + k
            for x in range(self.pages(left), self.pages(L)):
                if self.valid(self.table[b][x]):
                    self.ref[self.table[b][x]] -= 1
                else:
                    status[b] = ST_BAD_PAGE
                self.table[b][x] = -1
            self.length[b] = left
        return status

    def fork(self, parent, group):
        B = len(self.length)
        table, length, status = [list(r) for r in self.table], list(self.length), [0] * B
        for b in range(B):
            base = b // group * group
            p = base + parent[b] if 0 <= parent[b] < group and base + parent[b] < B else -1
            if p < 0 and parent[b] != -1:
                status[b] |= ST_BAD_ID
            if p == b:
                continue
            for which, row in ((+1, p), (-1, b)):
                L = self.length[row] if row >= 0 else 0
                if not self.ok(L):
                    status[b] |= ST_BAD_LENGTH
                    L = 0
                held = self.table[row][:self.pages(L)] if row >= 0 else []
                for i in held:
                    if self.valid(i):
                        self.ref[i] += which
                    else:
                        status[b] |= ST_BAD_PAGE
                if which > 0:
                    table[b] = held + [-1] * (self.max_pages - len(held))
                    length[b] = L
        self.table, self.length = table, length
        return status

    def compact(self):
        n = len(self.ref)
        used = sum(r != 0 for r in self.ref)
        src = [i for i in range(used, n) if self.ref[i] != 0]
        dst = [i for i in range(used) if self.ref[i] == 0]
        to = list(range(n))
        for s, d in zip(src, dst):
            to[s], self.ref[d], self.ref[s] = d, self.ref[s], 0
        status = [0] * len(self.length)
        for b, L in enumerate(self.length):
            if not self.ok(L):
                status[b] = ST_BAD_LENGTH
                continue
            for x in range(self.pages(L)):
                if self.valid(self.table[b][x]):
                    self.table[b][x] = to[self.table[b][x]]
                else:
                    status[b] = ST_BAD_PAGE
        pad = [-1] * (n // 2 - len(src))
        return src + pad, dst + pad, len(src), status


def paged_attention(q, k_pages, v_pages, page_table, length, scale, n_query=None, window=0, sinks=0, row_status=None):
    """q [B, Q, Hq, D], pools [n_pages, page_size, H, D] (float64) -> out, lse, status."""
    B, Q, Hq, D = q.shape
    n_pages, page, H = k_pages.shape[:3]
    out, lse, status = np.zeros(q.shape), np.full((B, Q, Hq), -np.inf), np.zeros(B, dtype=np.int64)
    for b in range(B):
        n, nq = int(length[b]), Q if n_query is None else int(n_query[b])
        if row_status is not None and row_status[b]:
            status[b] = row_status[b]
            continue
        if not 0 <= n <= page_table.shape[1] * page or not 0 <= nq <= Q:
            status[b] = ST_BAD_LENGTH
            continue
        seen = []
        for j in range(nq):
            p = n - nq + j
            seen.append([x for x in range(p + 1) if window <= 0 or x > p - window or x < sinks])
        if any(not 0 <= page_table[b, x // page] < n_pages for s in seen for x in s):
            status[b] = ST_BAD_PAGE
            continue
        for j, at in enumerate(seen):
            if not at:
                continue
            ids, slots = page_table[b, [x // page for x in at]], [x % page for x in at]
            for h in range(Hq):
                hk = h // (Hq // H)
                s = scale * (k_pages[ids, slots, hk] @ q[b, j, h])
                m = s.max()
                if m == -np.inf:
                    continue
                e = np.exp(s - m)
                lse[b, j, h] = m + np.log(e.sum())
                out[b, j, h] = (e / e.sum()) @ v_pages[ids, slots, hk]
    return out, lse, status


def beam_select(logits, score, n, temperature=1.0, finished=None, pad=0):
    """logits [B, W, V], score [B, W] (float64) -> parent, token, score [B, n], status [B, W]."""
    B, W, V = logits.shape
    parent, token, best = np.full((B, n), -1), np.full((B, n), -1), np.full((B, n), -np.inf)
    status = np.zeros((B, W), dtype=np.int64)
    for b in range(B):
        keys = np.full((W, V), -np.inf)
        for w in range(W):
            if np.isnan(score[b, w]) or score[b, w] == np.inf:
                status[b, w] = ST_NONFINITE
                continue
            if score[b, w] == -np.inf:
                continue
            if finished is not None and finished[b, w]:
                keys[w, pad] = score[b, w]
                continue
            z = logits[b, w] / temperature
            if np.isnan(z).any() or (z == np.inf).any():
                status[b, w] = ST_NONFINITE
                continue
            m = z.max()
            if m == -np.inf:
                continue
            keys[w] = score[b, w] + ((z - m) - np.log(np.exp(z - m).sum()))
        flat = keys.reshape(-1)
        order = np.argsort(-flat, kind="stable")[:n]
        for i, at in enumerate(order):
            if flat[at] > -np.inf:
                parent[b, i], token[b, i], best[b, i] = at // V, at % V, flat[at]
    return parent, token, best, status
