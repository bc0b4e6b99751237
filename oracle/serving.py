"""CPU oracle for the serving operations over a paged cache (numpy, float64).

TEST INFRASTRUCTURE ONLY (like the rest of ``oracle``).  Standard definitions, written out from the
formulas in include/laq.h, on float64 arrays (the caller converts from the 16-bit types, exactly):

* ``paged_append``    -- per-head RMSNorm of q and k, rotary embedding, the slots of the new tokens;
* ``paged_attention`` -- causal grouped-query attention of each request's new tokens over its pages;
* ``sample_bounds``   -- for each token the range of u that draws it, by weights in 64 bits.
"""
import math

import numpy as np

from .decoder import rope


def rows_of(q_start, kv_len):
    """(row, request, position) of every row of the batch."""
    for b in range(len(kv_len)):
        n = q_start[b + 1] - q_start[b]
        for i in range(n):
            yield q_start[b] + i, b, kv_len[b] - n + i


def paged_append(qkv, table, q_start, kv_len, Hq, Hkv, page_size, q_w, k_w, theta, eps, D=128):
    """(q [T, Hq, D], {(page, head, slot): (k, v)}) in float64; q_w or k_w None: no norm."""
    T = qkv.shape[0]
    heads = qkv.reshape(T, Hq + 2 * Hkv, D)

    def norm(x, w):
        return x if w is None else x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * w

    q, stored = np.zeros((T, Hq, D)), {}
    for row, b, p in rows_of(q_start, kv_len):
        q[row] = rope(norm(heads[row, :Hq], q_w), p, theta)
        if p < 0:
            continue
        k = rope(norm(heads[row, Hq:Hq + Hkv], k_w), p, theta)
        for g in range(Hkv):
            stored[int(table[b][p // page_size]), g, p % page_size] = (k[g],
                                                                      heads[row, Hq + Hkv + g])
    return q, stored


def paged_attention(q, k, v, table, q_start, kv_len, scale):
    """(out, A) [T, Hq, D]: out = sum_t P_t v_t, A = sum_t P_t |v_t|, P = softmax over t <= p;
    k, v [pages, Hkv, page_size, D]; a page outside the cache reads as zeros."""
    T, Hq, D = q.shape
    pages, Hkv, P, _ = k.shape
    G = Hq // Hkv
    out, A = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(kv_len)):
        n, L = q_start[b + 1] - q_start[b], kv_len[b]
        if n == 0 or L == 0:
            continue
        t = np.arange(L)
        page = np.asarray(table[b])[t // P]
        bad = (page < 0) | (page >= pages)
        page = np.where(bad, 0, page)
        ok = np.arange(L)[None] <= (L - n + np.arange(n))[:, None]      # [n, L]
        for g in range(Hkv):
            kk, vv = k[page, g, t % P].copy(), v[page, g, t % P].copy()
            kk[bad] = 0
            vv[bad] = 0
            for h in range(g * G, (g + 1) * G):
                s = np.where(ok, scale * (q[q_start[b]:q_start[b + 1], h] @ kk.T), -np.inf)
                top = s.max(1, keepdims=True)
                e = np.exp(s - np.where(top == -np.inf, 0, top))
                z = e.sum(1, keepdims=True)
                prob = e / np.where(z == 0, 1, z)
                out[q_start[b]:q_start[b + 1], h] = prob @ vv
                A[q_start[b]:q_start[b + 1], h] = prob @ np.abs(vv)
    return out, A


def sample_bounds(x, t=1.0, top_k=0, top_p=1.0, min_p=0.0, slack=0.0):
    """For one row of logits x [V] (float64) the kept set and each kept token's (low, high) of u:
    token v is drawn for low <= u < high.  Returns (kept indices ascending, low, high, share).
    ``slack`` moves the top_p target (for the two readings that rounding may take)."""
    x = np.where(np.isnan(x), -np.inf, x)
    V = len(x)
    order = np.lexsort((np.arange(V), -x))
    if not t > 0:
        order, w = order[:1], np.ones(1)
    else:
        top = x.max()
        with np.errstate(invalid="ignore"):
            w = np.where(x == top, 1.0, np.exp((x - top) / t))[order]
        if top_k > 0:
            order, w = order[:top_k], w[:top_k]
        if top_p < 1:
            cum = np.cumsum(w)
            n = int(np.sum(cum < (max(top_p, 0) + slack) * cum[-1])) + 1
            order, w = order[:n], w[:n]
        if min_p > 0:
            n = int(np.sum(w >= min(min_p, 1.0)))
            order, w = order[:n], w[:n]
    at = np.argsort(order)
    order, w = order[at], w[at] / math.fsum(w)
    high = np.cumsum(w)
    return order, high - w, high, w
