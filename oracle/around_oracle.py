"""The operators around the products in 64 bits, from their definitions -- TEST INFRASTRUCTURE, not product code.

Numpy arrays in, float64 arrays out; nothing of the HIP library is used.  Gradients follow the formulas, which the CPU tests
hold against differences of the forward functions.
"""
from __future__ import annotations

import math

import numpy as np

_M64 = (1 << 64) - 1
DROP_TENSOR = 4          # random-stream id of dropout


def drop_key(seed):
    z = (int(seed) + (DROP_TENSOR + 1) * 0x9E3779B97F4A7C15) & _M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & _M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & _M64
    z ^= z >> 31
    return z & 0xFFFFFFFF, z >> 32


def drop_factor(index, p, seed):
    """What element `index` (int64 array) of the stream is multiplied by: 0 or 65536 / (65536 - t)."""
    index = np.asarray(index, dtype=np.uint64)
    t = int(math.floor(65536.0 * p + 0.5))
    if t == 0:
        return np.ones(index.shape)
    k0, k1 = drop_key(seed)
    x = (index >> np.uint64(1)).astype(np.uint32) ^ np.uint32(k0)
    x ^= x >> np.uint32(16)
    x = x * np.uint32(0x7FEB352D)
    x ^= x >> np.uint32(15)
    x ^= np.uint32(k1)
    x = x * np.uint32(0x846CA68B)
    x ^= x >> np.uint32(16)
    half = np.where((index & np.uint64(1)) == 0, x & np.uint32(0xFFFF), x >> np.uint32(16))
    return np.where(half >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0)


def dropout(x, residual, p, seed):
    x = np.asarray(x, np.float64)
    f = drop_factor(np.arange(x.size).reshape(x.shape), p, seed)
    with np.errstate(invalid="ignore"):
        y = np.where(f == 0, 0.0, x * f)
    return y if residual is None else np.asarray(residual, np.float64) + y


# ---- activations ----

_erf = np.vectorize(math.erf, otypes=[np.float64])


def _sigmoid(z):
    return 0.5 * (1 + np.tanh(0.5 * z))


def act(z, kind):
    if kind == 1:
        return np.maximum(z, 0)
    if kind == 2:
        return z * _sigmoid(z)
    if kind == 3:
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    return z


def act_slope(z, kind):
    if kind == 1:
        return (z > 0).astype(np.float64)
    if kind == 2:
        s = _sigmoid(z)
        return s + z * s * (1 - s)
    if kind == 3:
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


# ---- group normalisation, x [Nb, P, C] ----

def _grouped(x, groups):
    Nb, P, C = x.shape
    return x.reshape(Nb, P, groups, C // groups)


def group_stats(x, groups, eps):
    g = _grouped(np.asarray(x, np.float64), groups)
    m = g.mean((1, 3))
    v = ((g - m[:, None, :, None]) ** 2).mean((1, 3))
    return m, 1 / np.sqrt(v + eps)


def group_norm_act(x, w, b, groups, eps, kind, p, seed):
    """-> y, mean, rstd"""
    x = np.asarray(x, np.float64)
    m, r = group_stats(x, groups, eps)
    xh = ((_grouped(x, groups) - m[:, None, :, None]) * r[:, None, :, None]).reshape(x.shape)
    y = act(xh * (1 if w is None else np.asarray(w, np.float64)) + (0 if b is None else np.asarray(b, np.float64)), kind)
    return y * drop_factor(np.arange(x.size).reshape(x.shape), p, seed), m, r


def group_norm_act_backward(dy, x, w, b, groups, eps, kind, p, seed):
    """-> dx, dw, db"""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    w = np.ones(x.shape[2]) if w is None else np.asarray(w, np.float64)
    b = np.zeros(x.shape[2]) if b is None else np.asarray(b, np.float64)
    m, r = group_stats(x, groups, eps)
    m, r = m[:, None, :, None], r[:, None, :, None]
    xh = ((_grouped(x, groups) - m) * r).reshape(x.shape)
    dz = dy * drop_factor(np.arange(x.size).reshape(x.shape), p, seed) * act_slope(xh * w + b, kind)
    dn, xg = _grouped(dz * w, groups), _grouped(xh, groups)
    dx = r * (dn - dn.mean((1, 3), keepdims=True) - xg * (dn * xg).mean((1, 3), keepdims=True))
    return dx.reshape(x.shape), (dz * xh).sum((0, 1)), dz.sum((0, 1))


# ---- attention map with a relative position bias, s [B, H, Q, K] ----

def rel_index(Q, K, grid_w):
    """[Q, K] number of the relative position of every key to every query"""
    r = np.empty((Q, K), np.int64)
    for q in range(Q):
        for k in range(K):
            if grid_w:
                h = K // grid_w
                dy, dx = k // grid_w - q // grid_w, k % grid_w - q % grid_w
                r[q, k] = (dy + h - 1) * (2 * grid_w - 1) + dx + grid_w - 1
            else:
                r[q, k] = k - q + Q - 1
    return r


def rel_count(Q, K, grid_w):
    return (2 * (K // grid_w) - 1) * (2 * grid_w - 1) if grid_w else Q + K - 1


def _rel_bias(table, buckets, rel):
    """[H, Q, K]: 0 where the bucket is none"""
    c = np.asarray(buckets)[rel]
    ok = (c >= 0) & (c < table.shape[0])
    return np.where(ok[None], np.asarray(table, np.float64)[np.where(ok, c, 0)].transpose(2, 0, 1), 0.0)


def rel_seen(B, Q, K, mask, causal):
    """[B, Q, K] truth values"""
    seen = np.ones((B, Q, K), bool)
    if causal:
        seen &= (np.arange(K)[None, :] <= np.arange(Q)[:, None] + K - Q)[None]
    if mask is not None:
        m = np.asarray(mask) != 0
        seen &= m[np.arange(B) % m.shape[0]]
    return seen


def _rel_map(s, table, buckets, mask, grid_w, causal, scale, rel):
    s = np.asarray(s, np.float64)
    B, H, Q, K = s.shape
    seen = np.broadcast_to(rel_seen(B, Q, K, mask, causal)[:, None], s.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(seen, s * scale + _rel_bias(table, buckets, rel)[None], -np.inf)
        top = z.max(-1, keepdims=True, initial=-np.inf)
        e = np.exp(z - np.where(top == -np.inf, 0.0, top))
        total = e.sum(-1, keepdims=True)
        return np.where(total == 0, 0.0, e / np.where(total == 0, 1.0, total)), z == -np.inf


def _map_factor(shape, p, seed):
    B, H, Q, K = shape
    Kp = (K + 7) // 8 * 8
    i = np.arange(B * H * Q)[:, None] * Kp + np.arange(K)[None, :]
    return drop_factor(i, p, seed).reshape(shape)


def rel_softmax(s, table, buckets, mask, grid_w, causal, scale, p, seed, rel=None):
    rel = rel_index(s.shape[2], s.shape[3], grid_w) if rel is None else rel
    pr, _ = _rel_map(s, table, buckets, mask, grid_w, causal, scale, rel)
    f = _map_factor(s.shape, p, seed)
    return np.where(f == 0, 0.0, pr * f)


def rel_softmax_backward(dP, s, table, buckets, mask, grid_w, causal, scale, p, seed, rel=None):
    """-> dS, dtable"""
    rel = rel_index(s.shape[2], s.shape[3], grid_w) if rel is None else rel
    pr, none = _rel_map(s, table, buckets, mask, grid_w, causal, scale, rel)
    f = _map_factor(s.shape, p, seed)
    with np.errstate(invalid="ignore"):
        dp = np.where(none | (f == 0), 0.0, np.asarray(dP, np.float64) * f)
        dz = np.where(none, 0.0, pr * (dp - (pr * dp).sum(-1, keepdims=True)))
    by_place = dz.sum(0).reshape(s.shape[1], -1)                        # [H, Q K]
    c = np.asarray(buckets)[rel].reshape(-1)
    dtable = np.zeros((table.shape[0], s.shape[1]))
    ok = (c >= 0) & (c < table.shape[0])
    for h in range(s.shape[1]):
        dtable[:, h] = np.bincount(c[ok], by_place[h][ok], table.shape[0])
    return dz * scale, dtable
