"""Plain fp64 definition of the operators on a paged cache (include/codecomp_cache.h), on the CPU.  Test infrastructure only; shares no
code with the library.  Values that come in bf16 or FP8 are handed in as fp64 numbers."""
from __future__ import annotations

import numpy as np


def frequencies(dim, base=10000.0, scaling="plain", factor=1.0, context=0.0, low=1.0, high=4.0):
    i = np.arange(dim // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (dim / (dim - 2))
    f = base ** (-2 * i / dim)
    if scaling == "linear":
        return f / factor
    if scaling == "wavelength":
        out = []
        for x in f:
            turns = context * x / (2 * np.pi)
            if turns >= high:
                out.append(x)
            elif turns <= low:
                out.append(x / factor)
            else:
                t = (turns - low) / (high - low)
                out.append((1 - t) * x / factor + t * x)
        return np.array(out)
    if scaling == "ramp":
        n = lambda turns: dim * np.log(context / (2 * np.pi * turns)) / (2 * np.log(base))  # noqa: E731
        a, b = max(np.floor(n(high)), 0), min(np.ceil(n(low)), dim - 1)
        t = np.clip((i - a) / max(b - a, 0.001), 0, 1)
        return t * f / factor + (1 - t) * f
    return f


def rotate(x, positions, freq, *, interleaved=False, inverse=False, magnitude=1.0):
    """x [T, H, d]; freq of the dim / 2 pairs.  Angles from whole positions in extended precision."""
    dim = 2 * len(freq)
    a = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(freq, dtype=np.longdouble)[None, :]
    a = np.asarray(np.remainder(a, 2 * np.longdouble(np.pi) + np.longdouble("1.2246467991473531772e-16") * 2), dtype=np.float64)
    if inverse:
        a = -a
    c, s = np.cos(a)[:, None, :], np.sin(a)[:, None, :]
    y = np.array(x, dtype=np.float64)
    i0, i1 = (np.arange(0, dim, 2), np.arange(1, dim, 2)) if interleaved else (np.arange(dim // 2), np.arange(dim // 2, dim))
    x0, x1 = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = magnitude * (x0 * c - x1 * s), magnitude * (x0 * s + x1 * c)
    return y


def place(table, r, row, page_size, n_pages):
    """(page, row in it), or None where there is none."""
    if row < 0 or row // page_size >= table.shape[1]:
        return None
    page = int(table[r, row // page_size])
    return (page, row % page_size) if 0 <= page < n_pages else None


def attend(q, k_pages, v_pages, table, kv_lens, cu_q, *, max_kv_len, causal=True, scale=None):
    """q [T, Hq, d], pages of one layer [n_pages, Hkv, page_size, d] (values, scales applied).  Returns out, lse, and for tolerances
    the weighted magnitudes sum_j p_j |v_j| and the largest sum_i |q_i k_ij| of every row."""
    T, Hq, d = q.shape
    n_pages, Hkv, ps, _ = k_pages.shape
    scale = scale or 1 / np.sqrt(d)
    out, lse = np.zeros((T, Hq, d)), np.full((T, Hq), -np.inf)
    spread, reach = np.zeros((T, Hq, d)), np.zeros((T, Hq))
    for r in range(len(kv_lens)):
        n = min(max(int(kv_lens[r]), 0), max_kv_len)
        rows = [(j, place(table, r, j, ps, n_pages)) for j in range(n)]
        held = [(j, p) for j, p in rows if p is not None]
        if not held or cu_q[r] == cu_q[r + 1]:
            continue
        slots, pages, at = (np.array(x) for x in ([j for j, _ in held], [p[0] for _, p in held], [p[1] for _, p in held]))
        tokens = np.arange(cu_q[r], cu_q[r + 1])
        sees = slots[None, :] <= n - cu_q[r + 1] + tokens[:, None] if causal else np.ones((len(tokens), len(slots)), bool)
        some = sees.any(axis=1)
        for h in range(Hq):
            kk, vv, qq = k_pages[pages, h // (Hq // Hkv), at], v_pages[pages, h // (Hq // Hkv), at], q[tokens, h]
            z = np.where(sees, scale * (qq @ kk.T), -np.inf)
            m = np.where(some, z.max(axis=1), 0.0)[:, None]
            p = np.exp(z - m)
            total = p.sum(axis=1, keepdims=True)
            with np.errstate(divide="ignore"):
                lse[tokens, h] = (m + np.log(total))[:, 0]
            p /= np.where(some[:, None], total, 1.0)
            out[tokens, h] = p @ vv
            spread[tokens, h] = p @ np.abs(vv)
            reach[tokens, h] = np.where(sees, scale * (np.abs(qq) @ np.abs(kk).T), 0.0).max(axis=1)
    return out, lse, spread, reach
