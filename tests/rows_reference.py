"""The operators on rows of channels in 64 bits, on the CPU, from their definitions (include/abl.h): block stores, the residual
step with its norms, the gated unit, weight gradients.  numpy only; nothing of the library is called."""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def blocks_of(C):
    return -(-C // 32)


def store_size(M, C, K):
    return -(-M * blocks_of(C) * (4 * K + 1) // 128) * 128


def blocked(x):
    M, C = x.shape
    out = np.zeros((M, blocks_of(C) * 32))
    out[:, :C] = x
    return out.reshape(M, -1, 32)


def scale_bytes(xb, K):
    """Scale bytes of blocks [M, B, 32]: by trial of the exponent, as the definition says it."""
    top = np.abs(xb).max(-1, initial=0.0)
    bad = ~np.isfinite(xb).all(-1)
    limit = 127.5 if K == 8 else 7.0
    e = np.full(top.shape, -119)
    for _ in range(260):
        more = ~bad & (np.ldexp(top, -e) >= limit)
        if not more.any():
            break
        e = e + more
    return np.where(bad, 255, e + 127).astype(np.uint8)


def nearest_codes(y, K):
    """Codes (as bytes / nibbles) of y = x 2^-e, nearest value of the type, ties to even."""
    if K == 8:
        return np.rint(y).astype(np.int64) & 255
    a = np.abs(y)
    d = np.abs(a[..., None] - E2M1)
    best = d.min(-1, keepdims=True)
    near = d == best                      # one value, or two neighbours at a tie: the even index is taken
    first = near.argmax(-1)
    tie = near.sum(-1) == 2
    i = np.where(tie & (first % 2 == 1), first + 1, first)
    return i + 8 * np.signbit(y)


def pack(x, K, byte=None):
    """The store's bytes of x [M, C] (float64 holding the values of the tensor); byte: with these scales."""
    M, C = x.shape
    xb = blocked(x)
    byte = scale_bytes(xb, K) if byte is None else byte
    bad = byte == 255
    y = np.where(bad[..., None], 0.0, np.ldexp(np.where(bad[..., None], 0.0, xb), -(byte.astype(np.int64)[..., None] - 127)))
    codes = nearest_codes(y, K)
    if K == 4:
        codes = codes[..., 0::2] + 16 * codes[..., 1::2]
    out = np.zeros(store_size(M, C, K), np.uint8)
    raw = np.concatenate([codes.astype(np.uint8).ravel(), byte.ravel()])
    out[: raw.size] = raw
    return out


def unpack(store, M, C, K):
    """The values that a store stands for, float64 [M, C]."""
    B = blocks_of(C)
    n = M * B * 4 * K
    byte = store[n: n + M * B].astype(np.int64).reshape(M, B, 1)
    if K == 8:
        v = store[:n].view(np.int8).astype(np.float64)
    else:
        c = np.stack([store[:n] & 15, store[:n] >> 4], -1)
        v = np.where(c > 7, -1.0, 1.0) * E2M1[c & 7]
    v = np.ldexp(v.reshape(M, B, 32), byte - 127)
    return np.where(byte == 255, np.nan, v).reshape(M, 32 * B)[:, :C]


def norm(x, eps, center):
    if center:
        x = x - x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt((x * x).mean(1) + eps)
    return x * rstd[:, None], rstd


def norm_gradient(v, y, rstd, center):
    out = v - y * (v * y).mean(1, keepdims=True)
    return rstd[:, None] * (out - v.mean(1, keepdims=True) if center else out)


def gate_rows_of(gate, rows, M):
    return gate[np.arange(M) // rows]


def step_forward(r, b, gate, rows, w_post, w_pre, alpha, beta, eps, center):
    """r', n and what is stored: y = N(b) (or b), z = N(r'), with their rstd (None where there is none)."""
    y, rstd_b, p = None, None, None
    if b is not None:
        y, p = b, b
        if w_post is not None:
            y, rstd_b = norm(b, eps, center)
            p = y * w_post
        if gate is not None:
            p = p * gate_rows_of(gate, rows, len(r))
    r2 = alpha * r + (beta * p if p is not None else 0.0)
    z, rstd_n = norm(r2, eps, center)
    return dict(r=r2, n=z * w_pre, y=y, z=z, rstd_b=rstd_b, rstd_n=rstd_n)


def step_backward(dn, dr_out, y, rstd_b, z, rstd_n, gate, rows, w_post, w_pre, alpha, beta, center, has_b=True):
    M = len(dn)
    D = norm_gradient(dn * w_pre, z, rstd_n, center)
    if dr_out is not None:
        D = D + dr_out
    out = dict(dr=alpha * D, dw_pre=(dn * z).sum(0))
    if not has_b:
        return out
    e = beta * D
    if gate is not None:
        G = -(-M // rows)
        t = e * (y * w_post if w_post is not None else y)
        out["dgate"] = np.stack([t[g * rows: (g + 1) * rows].sum(0) for g in range(G)])
        e = e * gate_rows_of(gate, rows, M)
    if w_post is not None:
        out["dw_post"] = (e * y).sum(0)
        e = norm_gradient(e * w_post, y, rstd_b, center)
    out["db"] = e
    return out


def act(g, kind):
    """act(g) and its derivative; kind 0: SiLU, 1: GELU in its tanh form."""
    with np.errstate(over="ignore"):
        if kind == 0:
            s = 1 / (1 + np.exp(-g))
            return g * s, s + g * s * (1 - s)
        k = np.sqrt(2 / np.pi)
        t = np.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)
