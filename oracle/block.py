"""Row-wise operators of a policy block, float64, from their formulas (test infrastructure).

  ffn_*      G = X Wg^T, U = X Wu^T, A = s(G) U, Y = A Wd^T and the gradients of sum(Y * dY)
  qk_*       root-mean-square norms per head and rotary positions, forward and backward
  norm_*     h = a x + b gate n(y), o = n(h) and the gradients of sum(h * dh) + sum(o * do)
  attend     attention of one query per head over keys and values
  keep_mask  the kept elements of a dropout whose 16-bit uniforms come from Philox4x32-10
             (Salmon et al., SC'11)
"""
import numpy as np
from scipy.special import ndtr


def activation(g, act):
    """s(g) and s'(g); act: 'silu' or 'gelu'."""
    with np.errstate(over="ignore"):
        if act == "silu":
            sig = 1.0 / (1.0 + np.exp(-g))
            return g * sig, sig + g * sig * (1.0 - sig)
        cdf = ndtr(g)
        return g * cdf, cdf + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)


def ffn_forward(X, Wg, Wu, Wd, act):
    g, u = X @ Wg.T, X @ Wu.T
    return (activation(g, act)[0] * u) @ Wd.T


def ffn_backward(dY, X, Wg, Wu, Wd, act):
    """dX, dWg, dWu, dWd."""
    g, u = X @ Wg.T, X @ Wu.T
    q, slope = activation(g, act)
    dA = dY @ Wd
    dG, dU = dA * u * slope, dA * q
    return dG @ Wg + dU @ Wu, dG.T @ X, dU.T @ X, dY.T @ (q * u)


def rope_angles(pos, R, theta):
    """[N][R/2] angles of positions counted from 0."""
    return np.asarray(pos, dtype=np.float64)[:, None] * theta ** (-2.0 * np.arange(R // 2) / R)


def turn(x, cos, sin, interleaved):
    """x [N][H][D] with its first 2 * cos.shape[1] dims turned in pairs."""
    R = 2 * cos.shape[1]
    y = np.array(x, dtype=np.float64)
    i = np.arange(R // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    c, s = cos[:, None], sin[:, None]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def qk_forward(x, gain, eps, cos, sin, interleaved):
    """x [N][H][D] -> normed, scaled and turned."""
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    return turn(x * r * gain, cos, sin, interleaved)


def qk_backward(dy, x, gain, eps, cos, sin, interleaved):
    """dx and the gain's gradient."""
    r = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    dn = turn(dy, cos, -sin, interleaved)
    dgain = np.sum(dn * x * r, axis=(0, 1))
    dn = dn * gain
    return r * (dn - x * r * r * np.mean(dn * x, axis=-1, keepdims=True)), dgain


def _rms(x, eps):
    return 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def norm_forward(x, y, gy, go, gate, a, b, eps, post):
    """h and o of rows x and, if y is not None, a branch y; gate [N] (0: the branch is left out)."""
    h = x
    if y is not None:
        shut = gate == 0
        n = np.where(shut[:, None], 0.0, y)
        n = n * (_rms(n, eps) if post else 1.0) * gy
        h = a * x + b * gate[:, None] * n
    return h, h * _rms(h, eps) * go


def norm_backward(do, dh, h, y, gy, go, gate, a, b, eps, post):
    """dx, dy, dgy, dgo, dgate; do or dh may be 0 (a scalar), y None."""
    r = _rms(h, eps)
    g = go * do
    dH = dh + r * (g - h * r * r * np.mean(g * h, axis=-1, keepdims=True))
    dgo = np.sum(do * h * r, axis=0)
    if y is None:
        return dH, None, None, dgo, None
    ry = _rms(y, eps) if post else np.ones((len(y), 1))
    dgate = b * np.sum(dH * y * ry * gy, axis=-1)      # (of a shut gate too)
    y = np.where((gate == 0)[:, None], 0.0, y)
    ry = _rms(y, eps) if post else ry
    dn = b * gate[:, None] * dH
    dy = gy * dn
    if post:
        dy = ry * (dy - y * ry * ry * np.mean(dy * y, axis=-1, keepdims=True))
    return a * dH, dy, np.sum(dn * y * ry, axis=0), dgo, dgate


def attend(q, k, v, scale):
    """q [Hq][D], k and v [n][Hk][D] -> o [Hq][D] and lse [Hq]; no keys: zeros and -inf."""
    Hq, Hk = q.shape[0], k.shape[1]
    if len(k) == 0:
        return np.zeros_like(q), np.full(Hq, -np.inf)
    of = np.arange(Hq) // (Hq // Hk)
    s = scale * np.einsum("hd,jhd->hj", q, k[:, of])
    top = s.max(axis=1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(axis=1, keepdims=True)
    return np.einsum("hj,jhd->hd", e / total, v[:, of]), (top + np.log(total))[:, 0]


def philox4x32_10(counter, key):
    """counter [..., 4] and key (two words) -> [..., 4], all 32-bit values in uint64."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.asarray(counter[..., i], dtype=np.uint64) & low for i in range(4)]
    k = [int(key[0]) & 0xFFFFFFFF, int(key[1]) & 0xFFFFFFFF]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> half) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> half) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1)


def keep_cut(p):
    """K of p = K / 2^16."""
    return int(np.floor(65536.0 * p + 0.5))


def keep_mask(traj, pos, d, p, seed, step, site, traj_base=0):
    """[N][d] of truth values: column c of row i is kept."""
    traj, pos = np.asarray(traj, dtype=np.int64), np.asarray(pos, dtype=np.int64)
    blocks = (d + 7) // 8
    counter = np.zeros((len(traj), blocks, 4), dtype=np.uint64)
    counter[..., 0] = (site << 16) + np.arange(blocks)
    counter[..., 1] = (pos & 0xFFFFFFFF)[:, None]
    counter[..., 2] = ((traj + traj_base) & 0xFFFFFFFF)[:, None]
    counter[..., 3] = step
    w = philox4x32_10(counter, (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
    u = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=-1).reshape(len(traj), blocks * 8)
    return u[:, :d] >= keep_cut(p)
