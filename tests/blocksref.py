"""Plain forms, in 64 bits on the host, of the operators over pages and blocks: pages and slots, bounds of
blocks, the blocks a query takes, attention over listed blocks."""
from __future__ import annotations

import math

import numpy as np


def plan(table, pt, free, count, n_k, n_new, T):
    """The step of atf_plan_pages, row by row, on copies: a dict of its outputs."""
    table, free = [list(map(int, r)) for r in table], list(map(int, free))
    B, width = len(table), len(table[0])
    cap = width * pt
    pages = lambda n: -(-n // pt)
    n_k = [min(max(int(n), 0), cap) for n in n_k]
    top = min(max(int(count), 0), len(free))
    for b in range(B):
        if n_new[b] < 0:
            for page in table[b][:pages(n_k[b])]:
                if top < len(free):
                    free[top] = page
                    top += 1
    out, starts, first, stopped, refused, tokens = list(n_k), [0], [], False, 0, 0
    for b in range(B):
        m = max(int(n_new[b]), 0)
        if n_new[b] < 0:
            out[b] = 0
        fits = n_k[b] + m <= cap
        need = pages(n_k[b] + m) - pages(n_k[b]) if fits else 0
        tokens += m
        stopped = stopped or need > top or tokens > T
        first.append(-1)
        if m and fits and not stopped:
            first[b] = n_k[b]
            for i in range(need):
                top -= 1
                table[b][pages(n_k[b]) + i] = free[top]
            out[b] += m
        elif m:
            refused += 1
        starts.append(min(tokens, T))
    slots, rows, positions = [-1] * T, [-1] * T, [-1] * T
    for b in range(B):
        for t in range(starts[b], starts[b + 1]):
            if first[b] >= 0:
                p = first[b] + t - starts[b]
                page = table[b][p // pt]
                slots[t], rows[t], positions[t] = page * pt + p % pt if page >= 0 else -1, b, p
    return dict(block_table=np.array(table), free_pages=np.array(free), n_k_out=np.array(out),
                row_starts=np.array(starts), slots=np.array(slots, dtype=np.int64), token_rows=np.array(rows),
                positions=np.array(positions), counts=np.array([top, starts[-1], refused]))


def v_slot(t):
    """Slot of token t of a 16-token V block."""
    return 8 * (t // 4 % 2) + 4 * (t // 8) + t % 4


def put_k(pool, page, tok, k):
    """Key k [h, d] into a K pool [P, h, d/16, pt, 16]."""
    h, d = k.shape
    pool[page, :, :, tok, :8] = k[:, :d // 2].reshape(h, d // 16, 8)
    pool[page, :, :, tok, 8:] = k[:, d // 2:].reshape(h, d // 16, 8)


def put_v(pool, page, tok, v):
    pool[page, :, tok // 16, :, v_slot(tok % 16)] = v


def get_k(pool, page, tok):
    x = pool[page, :, :, tok]
    return np.concatenate([x[:, :, :8].reshape(x.shape[0], -1), x[:, :, 8:].reshape(x.shape[0], -1)], axis=1)


def row_keys(pool, table_row, pt, n):
    """Keys 0 .. n - 1 of a row, [n, h, d]."""
    P = pool.shape[0]
    return np.stack([get_k(pool, min(max(int(table_row[t // pt]), 0), P - 1), t % pt) for t in range(n)])


def row_values(pool, table_row, pt, n):
    P = pool.shape[0]
    return np.stack([pool[min(max(int(table_row[t // pt]), 0), P - 1), :, t % pt // 16, :, v_slot(t % 16)]
                     for t in range(n)])


def bounds(kpool, out, table, n_k, n_new, max_new, pt, bt):
    """atf_block_bounds on out [P, h, pt/bt, d/16, 2, 16], in place."""
    P, h, nc = kpool.shape[:3]
    cap = table.shape[1] * pt
    for b in range(len(n_k)):
        n = min(max(int(n_k[b]), 0), cap)
        m = min(max(int(n_new[b]), 0), max_new, n)
        if m == 0:
            continue
        for j in range((n - m) // bt, (n - 1) // bt + 1):
            page = min(max(int(table[b, j * bt // pt]), 0), P - 1)
            at = j * bt % pt
            x = kpool[page, :, :, at: at + min(bt, n - j * bt)]  # [h, nc, tokens, 16]
            out[page, :, at // bt, :, 0] = x.max(axis=2)  # (numpy's propagate NaN)
            out[page, :, at // bt, :, 1] = x.min(axis=2)
    return out


def pair_bounds(x):
    """[..., d/16, 16] as [..., 2, d/2]: first and second components of the pairs."""
    return np.stack([x[..., :8].reshape(x.shape[:-2] + (-1,)), x[..., 8:].reshape(x.shape[:-2] + (-1,))], axis=-2)


def scores(q, bnd, table_row, p, last, W, pt, bt):
    """Scores [h_kv, blocks] of one token's query q [h_q, d] for its row's blocks."""
    P, h_kv, per = bnd.shape[:3]
    h_q, d = q.shape
    n = last // bt + 1
    G, half = h_q // h_kv, d // 2
    out = np.empty((h_kv, n))
    qs = q.reshape(h_kv, G, 2, half)
    for j in range(n):
        page = min(max(int(table_row[j // per]), 0), P - 1)
        hi, lo = pair_bounds(bnd[page, :, j % per, :, 0]), pair_bounds(bnd[page, :, j % per, :, 1])
        near, far = p - min(j * bt + bt - 1, last), p - j * bt
        keep = W >= near
        with np.errstate(invalid="ignore"):
            u = np.maximum(qs, 0) * hi[:, None] + np.minimum(qs, 0) * lo[:, None]
            u = u[:, :, 0] + u[:, :, 1]
            cut = (W < far) & (u < 0)
            u = np.where(cut, 0.0, u)
            # fsum: correctly rounded, so that the order of two scores is the exact sums'
            s = np.array([[_sum(u[g, i][keep]) for i in range(G)] for g in range(h_kv)])
        out[:, j] = np.where(np.isnan(s).any(axis=1), np.nan, s.max(axis=1))
    return out


def _sum(x):
    return math.fsum(x) if np.isfinite(x).all() else float(np.sum(x))


def select(q, bnd, table, rows, positions, n_k, max_n_k, W, pt, bt, top, first, lastn, out):
    """atf_select_blocks on out [T, h_kv, top], in place; the smallest relative gap at a border."""
    for t in range(len(rows)):
        b = int(rows[t])
        if b < 0 or b >= len(n_k):
            continue
        p = int(positions[t])
        last = min(min(max(int(n_k[b]), 0), max_n_k) - 1, p)
        out[t] = -1
        if last < 0:
            continue
        s = scores(q[t], bnd, table[b], p, last, W, pt, bt)
        n = s.shape[1]
        for g in range(s.shape[0]):
            rank = sorted(range(n), key=lambda j: (0 if j < first or j >= n - lastn else 1 if math.isnan(s[g, j]) else 2,
                                                   0 if math.isnan(s[g, j]) else -s[g, j], j))
            # (forced blocks and those that are NaN go by their index alone)
            forced = sorted(j for j in range(n) if j < first or j >= n - lastn)
            rank = forced + [j for j in rank if j not in set(forced)]
            take = sorted(rank[:top])
            out[t, g, :len(take)] = take
    return out


def attend(q, kpool, vpool, table, rows, positions, n_k, lists, W, pt, bt, scale):
    """o [T, h_q, d], lse [T, h_q], and per token and head the sum of |weight * value| [T, h_q, d] and
    the largest sum of |q k| over a kept key; NaN in rows of padding."""
    T, h_q, d = q.shape
    h_kv = kpool.shape[1]
    G, half = h_q // h_kv, d // 2
    o, lse = np.full((T, h_q, d), np.nan), np.full((T, h_q), np.nan)
    mass, size = np.zeros((T, h_q, d)), np.zeros((T, h_q))
    cache = {}
    cap = table.shape[1] * pt
    for t in range(T):
        b = int(rows[t])
        if b < 0 or b >= len(n_k):
            continue
        n = min(max(int(n_k[b]), 0), cap)
        last = min(n - 1, int(positions[t]))
        if b not in cache:
            cache[b] = (row_keys(kpool, table[b], pt, n), row_values(vpool, table[b], pt, n)) if n else None
        for g in range(h_kv):
            toks = [x for j in lists[t, g] if j >= 0 and last >= 0 and j <= last // bt
                    for x in range(j * bt, min((j + 1) * bt, last + 1))]
            hs = slice(g * G, (g + 1) * G)
            if not toks:
                o[t, hs], lse[t, hs] = 0.0, -math.inf
                continue
            toks = np.array(toks)
            k, v = cache[b][0][toks, g].copy(), cache[b][1][toks, g]
            drop = (int(positions[t]) - toks)[:, None] > W[None, :]
            k[np.concatenate([drop, drop], axis=1)] = 0.0
            a = (q[t, hs] @ k.T) * scale
            size[t, hs] = (np.abs(q[t, hs]) @ np.abs(k).T).max(axis=1) * scale
            m = a.max(axis=1, keepdims=True)
            e = np.exp(a - m)
            l = e.sum(axis=1, keepdims=True)
            o[t, hs] = e @ v / l
            mass[t, hs] = e @ np.abs(v) / l
            lse[t, hs] = (m + np.log(l))[:, 0]
    return o, lse, mass, size
