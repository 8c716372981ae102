"""Rotary positions with several axes, and attention over bf16 rows with a window and sinks or with a tree, in fp64 numpy, from what
``include/vitcop.h`` states."""
import numpy as np


def rotary(x, position, inv_freq, axis, token=None, seq_len=None, inverse=False):
    """(turned, written): rows [B, H, N, d] in fp64, and which of them the call writes (bool [B, N])."""
    B, H, N, d = x.shape
    F = len(inv_freq)
    out, written = np.array(x, np.float64), np.zeros((B, N), bool)
    for b in range(B):
        for r in range(N):
            t = r if token is None else min(int(token[b, r]), position.shape[2] - 1)
            if t < 0 or (seq_len is not None and r >= seq_len[b]):
                continue
            written[b, r] = True
            # (whole turns dropped while the product still has its digits)
            at = position[np.clip(axis, 0, position.shape[0] - 1), b, t].astype(np.longdouble) * np.asarray(inv_freq, np.longdouble)
            theta = np.asarray(np.mod(at, 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))), np.float64)
            c, s = np.cos(theta), -np.sin(theta) if inverse else np.sin(theta)
            a, e = x[b, :, r, :F], x[b, :, r, F:2 * F]
            out[b, :, r, :F], out[b, :, r, F:2 * F] = a * c - e * s, e * c + a * s
    return out, written


def seen_rows(n, count, t, window=None, n_sink=0, tree=None):
    """bool [n]: the rows that query t of ``count`` over ``n`` rows sees; ``tree``: its word."""
    j, base = np.arange(n), n - count
    p = base + t
    if p < 0:
        return np.zeros(n, bool)
    if tree is None:
        return (j <= p) & ((j < n_sink) | (j > p - window))
    return (j < base) | ((j >= base) & ((int(tree) >> np.clip(j - base, 0, 63)) & 1 == 1))


def attention(q, K, V, length, count, scale, window=None, n_sink=0, tree=None):
    """(out, lse, size, logit): outputs of queries [B, Hq, Tq, d] over rows [B, H, N, d], with the sum of weight |v| and the largest of
    |scale| sum |q k| that a query sees; queries from ``count[b]`` on stay NaN."""
    B, Hq, Tq, d = q.shape
    R = Hq // K.shape[1]
    out, lse = np.full(q.shape, np.nan), np.full((B, Hq, Tq), np.nan)
    size, logit = np.zeros(q.shape), np.zeros((B, Hq, Tq))
    for b in range(B):
        n, m = int(np.clip(length[b], 0, K.shape[2])), int(np.clip(count[b], 0, Tq))
        for t in range(m):
            see = np.flatnonzero(seen_rows(n, m, t, window, n_sink, None if tree is None else tree[b, t]))
            for h in range(Hq):
                out[b, h, t], lse[b, h, t] = 0.0, -np.inf
                if len(see) == 0:
                    continue
                k, v = K[b, h // R, see], V[b, h // R, see]
                with np.errstate(invalid="ignore", over="ignore"):
                    z = scale * (k @ q[b, h, t])
                    top = z.max()
                    if top == -np.inf:
                        continue
                    p = np.exp(z - top)
                    out[b, h, t], lse[b, h, t] = p @ v / p.sum(), top + np.log(p.sum())
                    size[b, h, t] = p @ np.abs(v) / p.sum()
                    logit[b, h, t] = abs(scale) * (np.abs(k) @ np.abs(q[b, h, t])).max()
    return out, lse, size, logit
