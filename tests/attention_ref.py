"""The layers of an attention block in 64 bits on the CPU (NCHW numpy arrays), written from their formulas."""
import numpy as np


def group_norm(x, gamma, beta, groups, eps, act):
    N, C, H, W = x.shape
    g = x.astype(np.float64).reshape(N, groups, -1)
    mean = g.mean(2, keepdims=True)
    var = ((g - mean) ** 2).mean(2, keepdims=True)
    with np.errstate(all="ignore"):
        y = ((g - mean) / np.sqrt(var + eps)).reshape(N, C, H, W)
        if gamma is not None:
            y = y * gamma.astype(np.float64)[:, None, None]
        if beta is not None:
            y = y + beta.astype(np.float64)[:, None, None]
        if act == "relu":
            y = np.where(np.isnan(y), np.nan, np.maximum(y, 0.0))
        elif act == "silu":
            y = y / (1.0 + np.exp(-y))
    return y


def attention(q, k, v, heads, kv_heads, scale, cap=0.0, bias=None, q_extents=None, k_extents=None):
    """q: [N][heads*D][QH][QW], k, v: [N][kv_heads*D][KH][KW], bias: [heads][QH+KH-1][QW+KW-1]."""
    N, C, QH, QW = q.shape
    _, _, KH, KW = k.shape
    D = C // heads
    out = np.zeros((N, C, QH, QW))
    qy, qx = np.divmod(np.arange(QH * QW), QW)
    ky, kx = np.divmod(np.arange(KH * KW), KW)
    for n in range(N):
        rows, keys = np.ones(QH * QW, bool), np.ones(KH * KW, bool)
        if q_extents is not None:
            rows = (qy < q_extents[n, 0]) & (qx < q_extents[n, 1])
        if k_extents is not None:
            keys = (ky < k_extents[n, 0]) & (kx < k_extents[n, 1])
        if not keys.any() or not rows.any():
            continue
        for h in range(heads):
            j = h // (heads // kv_heads)
            a = q[n, h * D:(h + 1) * D].reshape(D, -1).astype(np.float64)[:, rows]
            b = k[n, j * D:(j + 1) * D].reshape(D, -1).astype(np.float64)[:, keys]
            c = v[n, j * D:(j + 1) * D].reshape(D, -1).astype(np.float64)[:, keys]
            x = a.T @ b * scale
            if cap:
                x = cap * np.tanh(x / cap)
            if bias is not None:
                dy = qy[rows][:, None] - ky[keys][None] + KH - 1
                dx = qx[rows][:, None] - kx[keys][None] + KW - 1
                x = x + bias[h].astype(np.float64)[dy, dx]
            top = x.max(1, keepdims=True)
            p = np.exp(x - np.where(np.isneginf(top), 0.0, top))
            total = p.sum(1, keepdims=True)
            y = np.where(total > 0, p, 0.0) / np.where(total > 0, total, 1.0)
            flat = out[n, h * D:(h + 1) * D].reshape(D, -1)
            flat[:, rows] = (y @ c.T).T
    return out


def adapted(x, w, b, down, up, ids, scale, relu, before=None):
    """x: [N][C][H][W], w: [K][C], down: [A][R][C], up: [A][K][R], ids: [N] (outside 0 .. A - 1: none)."""
    N, C, H, W = x.shape
    f = x.astype(np.float64).reshape(N, C, -1)
    y = np.einsum("kc,ncp->nkp", w.astype(np.float64), f)
    if b is not None:
        y += b.astype(np.float64)[:, None]
    for n in range(N):
        a = int(ids[n])
        if 0 <= a < down.shape[0]:
            s = 1.0 if scale is None else float(scale[a])
            y[n] += s * (up[a].astype(np.float64) @ (down[a].astype(np.float64) @ f[n]))
    y = y.reshape(N, -1, H, W)
    if before is not None:
        y = y + before.astype(np.float64)
    return np.maximum(y, 0.0) if relu else y
