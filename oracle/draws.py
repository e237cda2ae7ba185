"""Plain numpy versions of the draw and dispatch calls (include/hx.h: hx_sample, hx_route_requests, hx_kv_place,
hx_kv_release), written from their definitions, one row after the other, in 64 bits or more.  Test infrastructure:
they share no code with the library."""
from __future__ import annotations

import numpy as np

I32_MIN = -(1 << 31)


def sample_row(x, draw, T=1.0, k=0, p=1.0, q=0.0):
    """(pick, logp, kept) of one row.  x: int32 or floating scores; draw: a 64-bit whole number."""
    x = np.asarray(x)
    masked = x == I32_MIN if x.dtype == np.int32 else np.isnan(x) | (x == -np.inf)
    at = np.flatnonzero(~masked)
    T, p, q = float(T), float(p), float(q)
    if at.size == 0 or not (0.0 <= T < np.inf) or np.isnan(p) or np.isnan(q):
        return -1, -np.inf, 0
    v = x[at].astype(np.float64)
    m = v.max()
    if T == 0.0:
        return int(at[np.argmax(v == m)]), 0.0, 1
    with np.errstate(over="ignore", invalid="ignore"):  # +inf scores: inf - inf where v == m, taken as 0
        z = np.where(v == m, 0.0, (v - m) / T)
        w = np.exp(z).astype(np.longdouble)
    by = np.argsort(-v, kind="stable")
    K = min(k, at.size) if k > 0 else at.size
    kept = K
    if p < 1.0:
        run = np.cumsum(w[by[:K]])
        kept = min(kept, 1 + int((run < p * run[-1]).sum()))
    if q > 0.0:
        kept = min(kept, int((w >= q).sum()))
    kept = max(kept, 1)
    mine = np.sort(by[:kept])
    run = np.cumsum(w[mine])
    t = np.longdouble(int(draw) >> 11) * np.longdouble(2.0) ** -53 * run[-1]
    past = np.flatnonzero(run > t)
    j = mine[past[0]] if past.size else mine[np.flatnonzero(w[mine] > 0)[-1]]
    return int(at[j]), float(z[j] - np.log(run[-1])), kept


def sample(x, draws, T=None, k=None, p=None, q=None):
    """Every row of x [R, N]; parameters are arrays of R or None (off).  (pick int32, logp float64, kept int32)."""
    rows = [sample_row(x[r], int(draws[r]) & ((1 << 64) - 1), 1.0 if T is None else T[r], 0 if k is None else int(k[r]),
                       1.0 if p is None else p[r], 0.0 if q is None else q[r]) for r in range(len(x))]
    return (np.array([a for a, _, _ in rows], np.int32), np.array([b for _, b, _ in rows], np.float64),
            np.array([c for _, _, c in rows], np.int32))


def route(n_p, n_d, max_p, max_d, max_pd, flow, draws):
    """Routes and lists of one network's flow column: a dict of the six outputs (int32)."""
    n = len(draws)
    ok = 0 <= n_p <= max_p and 0 <= n_d <= max_d and n_p * n_d <= max_pd
    ends = np.cumsum(np.maximum(np.asarray(flow[:n_p * n_d], np.int64), 0)) if ok and n_p * n_d else np.zeros(0, np.int64)
    total = int(ends[-1]) if len(ends) else 0
    pre, dec = np.full(n, -1, np.int32), np.full(n, -1, np.int32)
    if total:
        for i, d in enumerate(draws):
            t = ((int(d) & ((1 << 64) - 1)) * total) >> 64
            pre[i], dec[i] = divmod(int(np.searchsorted(ends, t, side="right")), n_d)

    def lists(node, nodes):
        order = np.argsort(np.where(node < 0, nodes, node), kind="stable").astype(np.int32)
        return order, np.concatenate([[0], np.cumsum([(node == k).sum() for k in range(nodes)])]).astype(np.int32)
    po, pb = lists(pre, max_p)
    do, db = lists(dec, max_d)
    return dict(prefill=pre, decode=dec, p_order=po, p_base=pb, d_order=do, d_base=db)


def _free(base, count, r):
    return int(np.clip(count[r], 0, max(0, base[r + 1] - base[r])))


def place(block_size, base, free_list, free_count, table, max_blocks, replica, held, n_new, slots):
    """table and slots are changed in place; returns (tok_base, placed, held_out, free_out)."""
    R, n = len(free_count), len(replica)
    left = [_free(base, free_count, r) for r in range(R)]
    closed = [False] * R
    tok, placed, out = np.zeros(n + 1, np.int64), np.zeros(n, np.uint8), np.asarray(held, np.int32).copy()
    for i in range(n):
        h, new, r = int(held[i]), int(n_new[i]), int(replica[i])
        add = max(new, 0)
        tok[i + 1] = tok[i] + add
        here = slice(min(int(tok[i]), len(slots)), min(int(tok[i + 1]), len(slots)))
        b0, b1 = -(-h // block_size), -(-(h + add) // block_size)
        ok = (0 <= r < R and h >= 0 and new >= 0 and h + add < 1 << 31 and b1 <= max_blocks
              and tok[i + 1] <= len(slots))
        if ok and b1 > b0 and (closed[r] or b1 - b0 > left[r]):
            closed[r], ok = True, False
        if not ok:
            slots[here] = -1
            continue
        top = int(base[r]) + left[r]
        table[i, b0:b1] = free_list[top - (b1 - b0):top][::-1]
        left[r] -= b1 - b0
        placed[i], out[i] = 1, h + add
        pos = np.arange(h, h + add)
        slots[here] = table[i, pos // block_size].astype(np.int64) * block_size + pos % block_size
    return tok, placed, out, np.array(left, np.int32)


def release(block_size, base, free_list, free_count, table, max_blocks, replica, held, done):
    """free_list is changed in place; returns (held_out, free_out)."""
    R, n = len(free_count), len(replica)
    count = [_free(base, free_count, r) for r in range(R)]
    closed = [False] * R
    out = np.asarray(held, np.int32).copy()
    for i in range(n - 1, -1, -1):
        h, r = int(held[i]), int(replica[i])
        nb = -(-h // block_size)
        if not done[i] or not 0 <= r < R or h < 0 or nb > max_blocks:
            continue
        if nb and (closed[r] or count[r] + nb > base[r + 1] - base[r]):
            closed[r] = True
            continue
        to = int(base[r]) + count[r]
        free_list[to:to + nb] = table[i, :nb][::-1]
        count[r] += nb
        out[i] = 0
    return out, np.array(count, np.int32)
