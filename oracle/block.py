"""Row-wise operators of a policy block, float64, from their formulas (test infrastructure).

  ffn_*      G = X Wg^T, U = X Wu^T, A = s(G) U, Y = A Wd^T and the gradients of sum(Y * dY)
  qk_*       root-mean-square norms per head and rotary positions, forward and backward
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
