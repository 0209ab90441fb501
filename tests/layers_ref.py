"""The layers in 64 bits on the host, from their definitions: linear attention
position by position, layer norm through its statistics, AdamW value by value.
Each also returns what its rounding error scales with: the same sums over
absolute values."""
import math

import numpy as np


def attention(q, k, v, log_decay, scale, initial=None, lengths=None):
    """q [B,T,Hq,Dk], k [B,T,Hkv,Dk], v [B,T,Hkv,Dv] -> (o, final, |o|, |final|)."""
    B, T, Hq, Dk = q.shape
    Hkv, Dv = v.shape[2:]
    G = Hq // Hkv
    gamma = np.exp(log_decay.astype(np.float64))[:, None, None]
    o, oa = np.zeros((B, T, Hq, Dv)), np.zeros((B, T, Hq, Dv))
    final = np.zeros((B, Hkv, Dk, Dv)) if initial is None else initial.astype(np.float64).copy()
    fa = np.abs(final)
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        S, A = final[b], fa[b]
        for t in range(n):
            kv = k[b, t][:, :, None] * v[b, t][:, None, :]
            S = gamma * S + kv
            A = gamma * A + np.abs(kv)
            qq = q[b, t].reshape(Hkv, G, Dk)
            o[b, t] = scale * np.matmul(qq, S).reshape(Hq, Dv)
            oa[b, t] = abs(scale) * np.matmul(np.abs(qq), A).reshape(Hq, Dv)
        final[b], fa[b] = S, A
    return o, final, oa, fa


def attention_backward(do, q, k, v, log_decay, scale, initial=None, lengths=None, dfinal=None):
    """-> dict of dq, dk, dv, dinitial, and of the same sums over absolute values."""
    def run(do, q, k, v, scale, S0, dS1):
        B, T, Hq, Dk = q.shape
        Hkv, Dv = v.shape[2:]
        G = Hq // Hkv
        gamma = np.exp(log_decay.astype(np.float64))[:, None, None]
        dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
        dinitial = dS1.copy()
        for b in range(B):
            n = T if lengths is None else min(max(int(lengths[b]), 0), T)
            S, D = S0[b], dS1[b]
            for t in range(n):
                S = gamma * S + k[b, t][:, :, None] * v[b, t][:, None, :]
                g = do[b, t].reshape(Hkv, G, Dv)
                dq[b, t] = scale * np.matmul(g, S.transpose(0, 2, 1)).reshape(Hq, Dk)
            for t in reversed(range(n)):
                qq, g = q[b, t].reshape(Hkv, G, Dk), do[b, t].reshape(Hkv, G, Dv)
                D = D + scale * np.matmul(qq.transpose(0, 2, 1), g)
                dk[b, t] = np.matmul(D, v[b, t][:, :, None])[:, :, 0]
                dv[b, t] = np.matmul(k[b, t][:, None, :], D)[:, 0]
                D = gamma * D
            dinitial[b] = D
        return dict(dq=dq, dk=dk, dv=dv, dinitial=dinitial)
    f = np.float64
    zeros = np.zeros((q.shape[0], k.shape[2], q.shape[3], v.shape[3]))
    args = [x.astype(f) for x in (do, q, k, v)]
    S0 = zeros if initial is None else initial.astype(f)
    dS1 = zeros if dfinal is None else dfinal.astype(f)
    return run(*args, scale, S0, dS1), run(*(np.abs(x) for x in args), abs(scale), np.abs(S0), np.abs(dS1))


def norm(x, w, b, eps):
    """-> (y, xhat, mean, rstd)."""
    x = x.astype(np.float64)
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    xhat = (x - mean) * rstd
    y = xhat * (1.0 if w is None else w.astype(np.float64)) + (0.0 if b is None else b.astype(np.float64))
    return y, xhat, mean[:, 0], rstd[:, 0]


def norm_backward(dy, x, w, eps):
    _, xhat, _, rstd = norm(x, None, None, eps)
    dy = dy.astype(np.float64)
    g = dy * (1.0 if w is None else w.astype(np.float64))
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, decay):
    """One step in 64 bits -> (p, m, v)."""
    p, g, m, v = (x.astype(np.float64) for x in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * decay) - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p, m, v


def decode_moments(m, v, m_scale, v_scale, block=256):
    """The values that 8-bit moments stand for."""
    mc, vc = m.astype(np.float64).reshape(-1, block), v.astype(np.float64).reshape(-1, block)
    mf = np.sign(mc) * (mc / 127.0) ** 2 * m_scale.astype(np.float64)[:, None]
    vf = (vc / 255.0) ** 4 * v_scale.astype(np.float64)[:, None]
    return mf.reshape(-1), vf.reshape(-1)


def unit(dtype: str) -> float:
    """The largest relative error of one rounding to the type."""
    return {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}[dtype]  # significands of 24 and 8 bits


def attention_bound(value, magnitude, dtype, terms):
    """How far an output may be off: its own rounding; with bf16 one rounding of
    each product's formed operand (a masked score, or the state that is read);
    and `terms` fp32 roundings of what is summed."""
    u = unit(dtype)
    formed = 1.02 * u if dtype == "bf16" else 0.0
    return u * np.abs(value) + (formed + terms * 2.0 ** -24) * magnitude + 1e-37


def state_bound(magnitude, dtype, terms):
    """States are sums in fp32; with bf16 a decayed operand is held in two bf16 parts, 2^-17 of it left out."""
    return ((2.0 ** -17 if dtype == "bf16" else 0.0) + terms * 2.0 ** -24) * magnitude + 1e-37


def attention_terms(T, Dk, Dv):
    """fp32 roundings on the way of one summand into an output: sums over the head, the
    positions and the state's steps, each decay a rounded power."""
    return Dk + Dv + 2 * T + 32


def ulps(n):
    return n * 2.0 ** -24


def finite_difference(f, x, d, h):
    """Central difference of f at x along d."""
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def log_decays(heads, lo=3.0, hi=10.0):
    bits = np.linspace(lo, hi, heads) if heads > 1 else np.array([4.0])
    return np.log1p(-np.exp2(-bits)).astype(np.float32)


def default_scale(d):
    return 1.0 / math.sqrt(d)
