"""The K/V cache in 4 bits and the attention over it, in fp64 numpy, from the format that ``include/vitcop.h`` states."""
import numpy as np

GROUP = BLOCK = 32


def round_bf16(x):
    """The nearest bf16 (ties to even) of fp64 values, as fp64."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
        step = np.ldexp(1.0, np.maximum(e - 8, -133))
        r = np.where(np.isfinite(x), np.rint(x / step) * step, x)
        return np.where(np.abs(r) >= 2.0 ** 128, np.sign(r) * np.inf, r)


def quantise(x):
    """(s, m, code) of rows [..., d] of bf16 values: fp64 [..., G], fp64 [..., G], int [..., G, 32]."""
    x = np.asarray(x, np.float64)
    x = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    with np.errstate(invalid="ignore", over="ignore"):
        lo, hi = x.min(-1), x.max(-1)                      # (numpy's pass NaN on)
        bad = ~((hi - lo) < 2.0 ** 128 * (1 - 2.0 ** -25))
        s = round_bf16((hi - lo) / 15)
        s = np.where(s < 2.0 ** -100, 0.0, s)
        m = round_bf16(lo + 8 * s)
        # (fp64 loses an element below 2^-53 of the centre, and with it the side of a border it is on.  The centre is a border, or 2^-10
        # of a step and more away from one, and at most 8.5 steps from 0: an element of 2^-40 of it is on the same side)
        least = np.ldexp(np.abs(m[..., None]), -40)
        x = np.where(x == 0, 0.0, np.copysign(np.maximum(np.abs(x), least), x))
        q = np.rint((x - m[..., None]) / np.where(s > 0, s, 1.0)[..., None])
        code = np.where(s[..., None] > 0, np.clip(q, -8, 7), 0.0) + 8
    s, m = np.where(bad, np.nan, s), np.where(bad, 0.0, m)
    return s, m, np.where(bad[..., None], 8.0, code).astype(np.int64)


def values(s, m, code):
    """What scales, centres and codes stand for: fp64 [..., d]."""
    v = m[..., None] + (code - 8) * s[..., None]
    return v.reshape(*v.shape[:-2], v.shape[-2] * GROUP)


def _bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def _float(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def pack(K, V):
    """bf16 values [B, H, Ncap, d] -> the cache's bytes [B, H, Ncap / 32, 40 d]."""
    B, H, N, d = np.shape(K)
    G, out = d // GROUP, np.zeros((B, H, N // BLOCK, 40 * d), np.uint8)
    for x, unit, at in ((K, 8, 0), (V, 4, 20 * d)):
        s, m, code = quantise(x)
        for r in range(BLOCK):
            for g in range(G):
                c = code[:, :, r::BLOCK, g]                # [B, H, blocks, 32]
                for e in range(GROUP):
                    byte = at + r * (d // 2) + (e // unit) * G * (unit // 2) + g * (unit // 2) + e % unit // 2
                    out[..., byte] |= (c[..., e] << (4 * (e % 2))).astype(np.uint8)
                for plane, where in ((s, 16 * d + 2 * (r * G + g)), (m, 18 * d + 2 * (r * G + g if unit == 8 else g * BLOCK + r))):
                    b = _bits(plane[:, :, r::BLOCK, g])
                    out[..., at + where], out[..., at + where + 1] = b & 255, b >> 8
    return out


def unpack(cache):
    """The cache's bytes -> ((s, m, code) of K, (s, m, code) of V), rows [B, H, Ncap, ..]."""
    B, H, blocks, width = cache.shape
    d = width // 40
    G, found = d // GROUP, []
    for unit, at in ((8, 0), (4, 20 * d)):
        s, m = np.zeros((B, H, blocks * BLOCK, G)), np.zeros((B, H, blocks * BLOCK, G))
        code = np.zeros((B, H, blocks * BLOCK, G, GROUP), np.int64)
        for r in range(BLOCK):
            for g in range(G):
                for e in range(GROUP):
                    byte = at + r * (d // 2) + (e // unit) * G * (unit // 2) + g * (unit // 2) + e % unit // 2
                    code[:, :, r::BLOCK, g, e] = cache[..., byte] >> (4 * (e % 2)) & 15
                for plane, where in ((s, 16 * d + 2 * (r * G + g)), (m, 18 * d + 2 * (r * G + g if unit == 8 else g * BLOCK + r))):
                    plane[:, :, r::BLOCK, g] = _float(cache[..., at + where].astype(np.uint16) | cache[..., at + where + 1].astype(np.uint16) << 8)
        found.append((s, m, code))
    return found


def attention(q, K, V, length, scale, causal):
    """(out, lse) of queries [B, Hq, Tq, d] over values [B, H, N, d], the first ``length[b]`` rows of each sample."""
    B, Hq, Tq, d = q.shape
    H = K.shape[1]
    out, lse = np.zeros(q.shape), np.full((B, Hq, Tq), -np.inf)
    for b in range(B):
        n = int(min(max(length[b], 0), K.shape[2]))
        for h in range(Hq):
            k, v = K[b, h // (Hq // H), :n], V[b, h // (Hq // H), :n]
            for t in range(Tq):
                seen = max(0, n - Tq + t + 1) if causal else n
                if seen == 0:
                    continue
                z = scale * (k[:seen] @ q[b, h, t])
                top = z.max()
                p = np.exp(z - top)
                out[b, h, t], lse[b, h, t] = p @ v[:seen] / p.sum(), top + np.log(p.sum())
    return out, lse
