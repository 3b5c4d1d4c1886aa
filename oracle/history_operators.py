"""Double-precision definitions of the operators that keep a history between requests (numpy, test infrastructure):
linear attention with a decay per head, and the 8-bit history cache.  Written from the definitions, event by event;
nothing is shared with the CUDA path."""
import numpy as np

BLOCK = 64


# ---- linear attention ---------------------------------------------------------------------------
def linear_attention(q, k, v, log_decay, scale, state0=None, lengths=None):
    """q, k, v [B,T,H,d] -> o [B,T,H,d] (zeros behind a length), last state [B,H,d,d]."""
    B, T, H, d = q.shape
    o, last = np.zeros((B, T, H, d)), np.zeros((B, H, d, d))
    for b in range(B):
        for h in range(H):
            g = np.exp(float(log_decay[h]))
            S = np.zeros((d, d)) if state0 is None else state0[b, h].astype(np.float64).copy()
            for t in range(T if lengths is None else int(lengths[b])):
                S = g * S + np.outer(k[b, t, h], v[b, t, h])
                o[b, t, h] = scale * (q[b, t, h] @ S)
            last[b, h] = S
    return o, last


def linear_attention_backward(q, k, v, log_decay, scale, dO, state0=None, dstate=None, lengths=None):
    B, T, H, d = q.shape
    dq, dk, dv, ds0 = (np.zeros((B, T, H, d)) for _ in range(3)), None, None, np.zeros((B, H, d, d))
    dq, dk, dv = dq
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        for h in range(H):
            g = np.exp(float(log_decay[h]))
            S = np.zeros((d, d)) if state0 is None else state0[b, h].astype(np.float64).copy()
            for t in range(n):
                S = g * S + np.outer(k[b, t, h], v[b, t, h])
                dq[b, t, h] = scale * (S @ dO[b, t, h])
            R = np.zeros((d, d)) if dstate is None else dstate[b, h].astype(np.float64).copy()
            for t in range(n - 1, -1, -1):
                R = R + scale * np.outer(q[b, t, h], dO[b, t, h])
                dk[b, t, h] = R @ v[b, t, h]
                dv[b, t, h] = k[b, t, h] @ R
                R = g * R
            ds0[b, h] = R
    return dq, dk, dv, ds0


# ---- the 8-bit cache ----------------------------------------------------------------------------
def round_e4m3(x):
    """Nearest e4m3 value, ties to even; |x| <= 448, NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(np.where(np.isfinite(x), x, 1.0))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(x / step) * step


def scale_exponent(amax):
    e = -100
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return e


def power_at_or_above(scale):
    """Smallest e in -100 .. 120 with scale <= 2^e (120 where there is none: 448 * 2^120 is past what fp32 holds)."""
    e = -100
    while e < 120 and scale > 2.0 ** e:
        e += 1
    return e


def append(cache, scales, rows, start, counts=None):
    """In place: rows [B,T,H,d] into cache [B,H,N,d] (e4m3 values as floats) and scales [B,H,N/64].  Older rows of a block are
    rounded to its new scale from what they stand for."""
    B, T, H, d = rows.shape
    N = cache.shape[2]
    for b in range(B):
        n = T if counts is None else min(max(int(counts[b]), 0), T)
        p0 = int(start[b])
        if p0 < 0 or p0 >= N:
            continue
        p1 = min(p0 + n, N)
        for blk in range(p0 // BLOCK, -(-p1 // BLOCK)):
            lo, hi = max(p0, blk * BLOCK), min(p1, (blk + 1) * BLOCK)
            if lo >= hi:
                continue
            for h in range(H):
                x = rows[b, lo - p0:hi - p0, h].astype(np.float64)
                x = np.where(np.isfinite(x), x, np.nan)
                e = scale_exponent(np.nanmax(np.abs(x), initial=0.0))
                if lo > blk * BLOCK:
                    old = float(scales[b, h, blk])
                    e = max(e, power_at_or_above(old))
                    cache[b, h, blk * BLOCK:lo] = np.clip(round_e4m3(cache[b, h, blk * BLOCK:lo] * (old * 2.0 ** -e)), -448.0, 448.0)
                scales[b, h, blk] = 2.0 ** e
                cache[b, h, lo:hi] = round_e4m3(x * 2.0 ** -e)


def attention(q, k8, v8, k_scale, v_scale, lengths, scale, causal=False):
    """q [B,M,Hq,d] over the first lengths[b] rows of the cache -> o, and the same with |v| in the place of v."""
    B, M, Hq, d = q.shape
    H, N = k8.shape[1], k8.shape[2]
    o, size = np.zeros((B, M, Hq, d)), np.zeros((B, M, Hq, d))
    for b in range(B):
        n = min(max(int(lengths[b]), 0), N)
        for hq in range(Hq):
            h = hq * H // Hq
            K = k8[b, h, :n] * np.repeat(k_scale[b, h], BLOCK)[:n, None]
            V = v8[b, h, :n] * np.repeat(v_scale[b, h], BLOCK)[:n, None]
            for m in range(M):
                see = max(min(n, n - M + m + 1), 0) if causal else n
                if see == 0:
                    continue
                z = scale * (K[:see] @ q[b, m, hq].astype(np.float64))
                p = np.exp(z - z.max())
                p /= p.sum()
                o[b, m, hq], size[b, m, hq] = p @ V[:see], p @ np.abs(V[:see])
    return o, size
