"""One decode iteration over a paged key / value cache: page assignment, per-head norm with rotary embedding, attention of one new
token per request, and a Linear with 4-bit weights.  TEST INFRASTRUCTURE ONLY: plain numpy float64, one request, token and head at a
time where that is the plainest form.

Readings (none of these is in the paper; they serve its decoder-only models, Table 7, at ragged lengths): pages are handed out in the
order of the requests; RMSNorm / LayerNorm as in oracle.ops, per head; rotary pairs (i, i + rot/2), theta_i = base^(-2i/rot); softmax
scale given by the caller; weights (w - z) * s per group along K.
"""
import numpy as np


def page_table(cached, fresh, free_pages, n_free, table, page, n_pages, max_tokens):
    """Returns table, starts, lens, positions, slots, need (see sm_page_table)."""
    table = np.array(table)
    R, row = table.shape[0], table.shape[1] * page
    n_free = max(0, min(int(n_free), len(free_pages)))
    starts, lens = np.zeros(R + 1, int), np.zeros(R, int)
    positions, slots = np.full(max_tokens, -1), np.full(max_tokens, -1)
    need, t = 0, 0
    for r in range(R):
        c = min(max(int(cached[r]), 0), row)
        starts[r] = t
        lens[r] = c
        pages = -(-c // page)               # pages the request has
        complete = True
        for j in range(min(max(int(fresh[r]), 0), max_tokens - t)):
            p = c + j
            positions[t + j] = p
            if p >= row:
                continue
            if p == pages * page:           # the token opens a page
                if need < n_free:
                    table[r, pages] = free_pages[need]
                else:
                    complete = False
                need += 1
                pages += 1
            if complete:
                lens[r] = p + 1
                e = table[r, p // page]
                if 0 <= e < n_pages:
                    slots[t + j] = e * page + p % page
        t += min(max(int(fresh[r]), 0), max_tokens - t)
    starts[R] = t
    return table, starts, lens, positions, slots, need


def head_norm(x, kind, gamma, beta, eps):
    """x [..., d]: the norm of every head."""
    if kind == "none":
        return x
    y = x - x.mean(-1, keepdims=True) if kind == "layer" else x
    y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gamma
    return y + beta if kind == "layer" else y


def rope(x, positions, rot, base):
    """x [T, heads, d] at positions [T]."""
    half = rot // 2
    theta = float(base) ** (-2.0 * np.arange(half) / max(rot, 1))
    ang = np.asarray(positions, np.float64)[:, None, None] * theta
    c, s = np.cos(ang), np.sin(ang)
    a, b = x[..., :half], x[..., half:rot]
    return np.concatenate([a * c - b * s, b * c + a * s, x[..., rot:]], -1)


def keys_of(pages, table_row, n, page):
    """The tokens [m, heads, d] that the first n places of a request hold, in order; places of pages outside the pool left out."""
    out = []
    for p in range(n):
        e = table_row[p // page]
        if 0 <= e < pages.shape[0]:
            out.append(pages[e, p % page])
    return np.array(out, np.float64).reshape(-1, *pages.shape[2:])


def paged_attention(q, k_pages, v_pages, table, lens, scale, want_bound=False):
    """q [R, hq, d], pages [n, page, hkv, d] -> o [R, hq, d], lse [R, hq]; with want_bound also sum_j p_j |v_j| and the largest
    sum_i |q_i k_i| * |scale| of a key (what rounding errors scale with)."""
    R, hq, d = q.shape
    page, hkv = k_pages.shape[1:3]
    o, lse = np.zeros((R, hq, d)), np.full((R, hq), -np.inf)
    av, aw = np.zeros((R, hq, d)), np.zeros((R, hq, 1))
    for r in range(R):
        n = max(0, min(int(lens[r]), table.shape[1] * page))
        K, V = keys_of(k_pages, table[r], n, page), keys_of(v_pages, table[r], n, page)
        if len(K) == 0:
            continue
        for h in range(hq):
            kk, vv = K[:, h // (hq // hkv)], V[:, h // (hq // hkv)]
            w = kk @ q[r, h] * scale
            m = w.max()
            p = np.exp(w - m)
            lse[r, h] = m + np.log(p.sum())
            p /= p.sum()
            o[r, h] = p @ vv
            if want_bound:
                av[r, h] = p @ np.abs(vv)
                aw[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * abs(scale)
    return (o, lse, av, aw) if want_bound else (o, lse)


def unpack_w4(w, scales, zeros, group):
    """w [N, K/2] bytes -> W [N, K]."""
    N, K = w.shape[0], 2 * w.shape[1]
    W = np.zeros((N, K))
    W[:, 0::2], W[:, 1::2] = w & 15, w >> 4
    z = np.full((N, K // group), 8.0) if zeros is None else zeros.astype(np.float64)
    return (W - np.repeat(z, group, 1)) * np.repeat(scales, group, 1)


def linear_w4(x, w, scales, zeros, group, bias=None, residual=None, act="none"):
    from .ops import gelu
    y = x @ unpack_w4(w, scales, zeros, group).T
    if bias is not None:
        y = y + bias
    if act == "gelu":
        y = gelu(y)
    return y if residual is None else y + residual
