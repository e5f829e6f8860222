"""Plain fp64 definition of the operators for shared and evicted caches (include/codecomp_serve.h), on the CPU.  Test infrastructure only; shares no
code with the library.  Values that come in bf16 or FP8 are handed in as fp64 numbers."""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle as orc


def by_rows(pages):
    """Pages [n_pages, Hkv, page_size, d] as pages of one row."""
    n, H, ps, d = pages.shape
    return pages.transpose(0, 2, 1, 3).reshape(n * ps, H, 1, d)


def rows_table(table, page_size, n_pages, kv_lens, cu_groups=None, prefix_lens=None):
    """Table of pages of one row: the first rows of a request are those of the first request of its group."""
    out = np.full((len(kv_lens), max([int(n) for n in kv_lens] + [1])), -1, np.int64)
    for r, n in enumerate(kv_lens):
        lead, before = r, 0
        if cu_groups is not None:
            g = int(np.searchsorted(cu_groups, r, side="right")) - 1
            lead, before = int(cu_groups[g]), int(prefix_lens[g])
        for j in range(int(n)):
            p = orc.place(table, lead if j < before else r, j, page_size, n_pages)
            if p is not None:
                out[r, j] = p[0] * page_size + p[1]
    return out


def attend_shared(q, k_pages, v_pages, table, kv_lens, cu_q, cu_groups, prefix_lens, *, causal=True, scale=None):
    """As cache_oracle.attend; the shared rows lie before all new tokens."""
    t = rows_table(table, k_pages.shape[2], k_pages.shape[0], kv_lens, cu_groups, prefix_lens)
    return orc.attend(q, by_rows(k_pages), by_rows(v_pages), t, kv_lens, cu_q, max_kv_len=t.shape[1], causal=causal, scale=scale)


def attend_mass(q, lse, k_pages, table, kv_lens, cu_q, sums, *, first=None, decay=1.0, causal=True, scale=None):
    """sums [n_seqs, Hkv, width] of one layer.  Returns the new sums, what was added, and the largest sum_i |q_i k_ij| and |logit| and |lse| that a sum has met."""
    T, Hq, d = q.shape
    n_pages, Hkv, ps, _ = k_pages.shape
    G, scale = Hq // Hkv, scale or 1 / np.sqrt(d)
    out, added, reach = np.array(sums, dtype=np.float64), np.zeros_like(sums, dtype=np.float64), np.zeros_like(sums, dtype=np.float64)
    for r in range(len(kv_lens)):
        n, nq = int(kv_lens[r]), int(cu_q[r + 1] - cu_q[r])
        if nq == 0:
            continue
        f = max(int(first[r]), 0) if first is not None else 0
        for j in range(f, n):
            p = orc.place(table, r, j, ps, n_pages)
            tokens = np.arange(max(0, j - (n - nq)) if causal else 0, nq) + cu_q[r]
            old = j < n - nq if causal else True
            for h in range(Hkv):
                add = 0.0
                if p is not None and len(tokens):
                    k = k_pages[p[0], h, p[1]]
                    qq, l = q[tokens, h * G:(h + 1) * G], lse[tokens, h * G:(h + 1) * G].astype(np.float64)
                    z = scale * (qq @ k)
                    live = ~np.isneginf(l)
                    with np.errstate(over="ignore", invalid="ignore"):
                        add = np.where(live, np.exp(z - np.where(live, l, 0.0)), 0.0).sum() / G
                    size = scale * (np.abs(qq) @ np.abs(k))
                    if live.any():
                        reach[r, h, j] = (size * (d + 16) + 2 * np.abs(z) + 2 * np.abs(np.where(live, l, 0.0)))[live].max()
                added[r, h, j] = add
                out[r, h, j] = (decay * sums[r, h, j] if old and decay != 0 else 0.0) + add
    return out, added, reach


def evict(sums, kv_lens, budgets, *, recent, max_budget, first=None):
    """sums [L, n_seqs, Hkv, width] (f32).  Returns kept [L, n_seqs, Hkv, max_budget] and the new lengths."""
    L, n_seqs, H, _ = sums.shape
    kept, lens = np.full((L, n_seqs, H, max_budget), -1, np.int32), np.zeros(n_seqs, np.int32)
    for r in range(n_seqs):
        n = int(kv_lens[r])
        f = min(max(int(first[r]), 0), n) if first is not None else 0
        b = min(max(int(budgets[r]), recent), max_budget)
        m = min(n - f, b)
        lens[r] = f + m
        for l in range(L):
            for h in range(H):
                if n - f <= b:
                    kept[l, r, h, :m] = np.arange(f, n)
                    continue
                rows = list(range(f, n - recent))
                x = [float(sums[l, r, h, j]) for j in rows]
                order = sorted(range(len(rows)), key=lambda i: (np.isnan(x[i]), 0.0 if np.isnan(x[i]) else -x[i], i))     # a stable order: ties by row
                best = [rows[i] for i in order[: m - recent]]
                kept[l, r, h, :m] = sorted(best) + list(range(n - recent, n))
    return kept, lens
