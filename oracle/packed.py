"""Float64 CPU oracle of the packed-sequence operators (test infrastructure only).

Rotary positions with several axes, softmax attention within the sequences of
a packed batch, and the gated feed-forward products, forward and backward,
written from their formulas in plain numpy.  Each function that a GPU kernel is
compared with also returns how far off a kernel may be that holds its sums in
fp32 and rounds to bf16 where the library says it does: elementwise bounds from
the magnitudes of the terms, in the unit roundoffs of bf16 (2^-8, relative to
the value) and of fp32 (2^-24).
"""

import numpy as np

from .encoder_layer import gelu, gelu_grad

__all__ = ["rope", "rope_bound", "packed_attention_fwd", "packed_attention_bwd", "glu_fwd", "glu_bwd", "glu_act",
           "glu_act_grad"]

BF16, FP32 = 2.0 ** -8, 2.0 ** -24


# ------------------------------------------------------------------ rotary positions

def rope(x, heads, kv_heads, d, pos, inv_freq, sections, interleaved, back=False):
    """x [M, (heads + 2 kv_heads) d] with every pair of a query or key vector
    turned by pos[row, axis] * inv_freq[pair] (back: by its negative)."""
    out = np.array(x, dtype=np.float64)
    v = out.reshape(out.shape[0], heads + 2 * kv_heads, d)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    for i, a in enumerate(axis):
        ang = pos[:, a].astype(np.float64) * np.float64(inv_freq[i]) * (-1.0 if back else 1.0)
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
        qk = slice(0, heads + kv_heads)
        a0, b0 = v[:, qk, lo].copy(), v[:, qk, hi].copy()
        v[:, qk, lo], v[:, qk, hi] = a0 * c - b0 * s, a0 * s + b0 * c
    return out


def rope_bound(x, ref, heads, kv_heads, d, pos, inv_freq, sections, interleaved):
    """One rounding to bf16; before it each result is two products with cos and
    sin off by 16 fp32 roundoffs at most (the angle's fraction of a turn times
    2 pi, and the functions), and three fp32 operations.  Far angles, formed in
    64 bits, add four of those roundoffs of their size.  Copies are exact."""
    v = np.abs(np.asarray(x, dtype=np.float64)).reshape(x.shape[0], heads + 2 * kv_heads, d)
    size = np.zeros_like(v)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    for i, a in enumerate(axis):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + d // 2)
        both = v[:, :heads + kv_heads, lo] + v[:, :heads + kv_heads, hi]
        far = 4 * 2.0 ** -53 * np.abs(pos[:, a] * np.float64(inv_freq[i]))[:, None]
        size[:, :heads + kv_heads, lo] = size[:, :heads + kv_heads, hi] = both * (19 * FP32 + far)
    err = size.reshape(ref.shape)
    return (BF16 * np.abs(ref) + err * (1 + BF16)) * (err > 0)


# ------------------------------------------------------------------ attention

def _heads(qkv, heads, kv, d):
    v = np.asarray(qkv, dtype=np.float64).reshape(qkv.shape[0], heads + 2 * kv, d)
    return v[:, :heads], v[:, heads:heads + kv], v[:, heads + kv:]


def _seen(n, causal):
    return np.tril(np.ones((n, n), dtype=bool)) if causal else np.ones((n, n), dtype=bool)


def packed_attention_fwd(qkv, cu, heads, kv_heads, d, causal):
    """(o, lse, o's bound, lse's bound); rows of no sequence are NaN."""
    T, g, scale = qkv.shape[0], heads // kv_heads, 1.0 / np.sqrt(d)
    q, k, v = _heads(qkv, heads, kv_heads, d)
    o = np.full((T, heads, d), np.nan)
    lse = np.full((heads, T), np.nan)
    ob, lb = o.copy(), lse.copy()
    for b, e in zip(cu[:-1], cu[1:]):
        n = e - b
        seen = _seen(n, causal)
        for h in range(heads):
            if n == 0:
                continue
            qh, kh, vh = q[b:e, h], k[b:e, h // g], v[b:e, h // g]
            s = np.where(seen, qh @ kh.T * scale, -np.inf)
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            total = p.sum(1, keepdims=True)
            p /= total
            o[b:e, h] = p @ vh
            lse[h, b:e] = (m + np.log(total))[:, 0]
            # a logit is off by its fp32 sum over d, its scaling and its
            # difference from the maximum; so is, relatively, its weight
            size = (np.abs(qh) @ np.abs(kh).T * scale * seen).max(1, keepdims=True)
            ds = FP32 * ((d + 4) * size + 4 * np.abs(m) + 8)
            weights = p @ np.abs(vh)
            # weights rounded to bf16 and summed, then one rounding; the sum of
            # n weights in fp32
            ob[b:e, h] = (BF16 + 2 * ds + 2 * (n + 16) * FP32) * weights + BF16 * np.abs(o[b:e, h]) * (1 + BF16)
            lb[h, b:e] = (2 * ds + (n + 16) * FP32)[:, 0] + 4 * FP32 * np.abs(lse[h, b:e])
    return o.reshape(T, heads * d), lse, ob.reshape(T, heads * d), lb


def packed_attention_bwd(qkv, cu, heads, kv_heads, d, causal, do):
    """(dqkv, its bound); rows of no sequence are NaN.  The bound takes in that a
    kernel is given o rounded to bf16 and lse in fp32."""
    T, g, scale = qkv.shape[0], heads // kv_heads, 1.0 / np.sqrt(d)
    q, k, v = _heads(qkv, heads, kv_heads, d)
    do = np.asarray(do, dtype=np.float64).reshape(T, heads, d)
    o, lse, ob, lb = packed_attention_fwd(qkv, cu, heads, kv_heads, d, causal)
    o, ob = o.reshape(T, heads, d), ob.reshape(T, heads, d)
    out = np.full((T, heads + 2 * kv_heads, d), np.nan)
    bound = out.copy()
    for b, e in zip(cu[:-1], cu[1:]):
        n = e - b
        if n == 0:
            continue
        seen = _seen(n, causal)
        out[b:e, heads:] = bound[b:e, heads:] = 0.0
        for h in range(heads):
            j = h // g
            qh, kh, vh, dh = q[b:e, h], k[b:e, j], v[b:e, j], do[b:e, h]
            p = np.where(seen, np.exp(qh @ kh.T * scale - lse[h, b:e][:, None]), 0.0)
            dp, D = dh @ vh.T, (dh * o[b:e, h]).sum(1, keepdims=True)
            ds = p * (dp - D)
            out[b:e, h] = ds @ kh * scale
            out[b:e, heads + j] += ds.T @ qh * scale
            out[b:e, heads + kv_heads + j] += p.T @ dh
            # relative error of a weight: its logit's and lse's
            size = np.abs(qh) @ np.abs(kh).T * scale
            rel = FP32 * ((d + 4) * size + 8 * np.abs(lse[h, b:e])[:, None] + 8) + lb[h, b:e][:, None]
            # dP's fp32 sum, and D from the rounded o
            ddp = (d + 4) * FP32 * (np.abs(dh) @ np.abs(vh).T)
            dD = (np.abs(dh) * (ob[b:e, h] + (d + 4) * FP32 * np.abs(o[b:e, h]))).sum(1, keepdims=True)
            eds = (BF16 + rel) * np.abs(ds) + p * (1 + rel) * (ddp + dD)
            # sums of n terms (over the shared heads, of g n) in fp32
            add = (g * n + 16) * FP32
            bound[b:e, h] = (eds + add * np.abs(ds)) @ np.abs(kh) * scale
            bound[b:e, heads + j] += (eds + add * np.abs(ds)).T @ np.abs(qh) * scale
            bound[b:e, heads + kv_heads + j] += ((BF16 + rel + add) * p).T @ np.abs(dh)
    bound += BF16 * (np.abs(out) + bound)
    return out.reshape(T, -1), bound.reshape(T, -1)


# ------------------------------------------------------------------ gated feed-forward

def glu_act(g, act):
    return gelu(g) if act == "gelu" else g / (1.0 + np.exp(-g))


def glu_act_grad(g, act):
    if act == "gelu":
        return gelu_grad(g)
    s = 1.0 / (1.0 + np.exp(-g))
    return s + g * s * (1.0 - s)


# The kernels' activations: off by a few fp32 roundoffs relative to |g| (the
# hardware's exponential and reciprocal, with an argument rounded relative to
# itself), and the normal distribution function by 1.5e-7 absolutely.
def _act_error(g):
    return (2e-7 + 16 * FP32) * (np.abs(g) + np.abs(g) ** 2 * np.exp(-np.abs(g)))


def glu_fwd(y, w_gu, b_gu, act):
    """(gu, h, gu's bound, h's bound)."""
    F, K = w_gu.shape[0] // 2, y.shape[1]
    b = np.zeros(2 * F) if b_gu is None else b_gu
    gu = y @ w_gu.T + b
    err = (K + 4) * FP32 * (np.abs(y) @ np.abs(w_gu).T + np.abs(b))
    g, u = gu[:, :F], gu[:, F:]
    a = glu_act(g, act)
    h = a * u
    # |act'| stays below 1.13
    ea = 1.13 * err[:, :F] + _act_error(g)
    hb = ea * (np.abs(u) + err[:, F:]) + np.abs(a) * err[:, F:]
    return gu, h, BF16 * (np.abs(gu) + err) + err, BF16 * (np.abs(h) + hb) + hb


def glu_bwd(dout, w_2, gu, act):
    """(dgu, its bound) from the saved gu as it is."""
    F, K = w_2.shape[1], w_2.shape[0]
    dh = dout @ w_2
    err = (K + 4) * FP32 * (np.abs(dout) @ np.abs(w_2))
    g, u = gu[:, :F], gu[:, F:]
    a, da = glu_act(g, act), glu_act_grad(g, act)
    dgu = np.concatenate([dh * u * da, dh * a], 1)
    e_da = (4e-7 + 16 * FP32) * (1 + np.abs(g))
    eb = np.concatenate([err * np.abs(u * da) + (np.abs(dh) + err) * np.abs(u) * (e_da + 2 * FP32),
                         err * np.abs(a) + (np.abs(dh) + err) * (_act_error(g) + FP32 * np.abs(a))], 1)
    return dgu, BF16 * (np.abs(dgu) + eb) + eb
