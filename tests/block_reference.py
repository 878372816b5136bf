"""The operators of the feed-forward block from their definitions, in numpy and 64 bits, and how far fp32
sums and the stated roundings may be from them."""
import math

import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
HALF16 = 2.0 ** -8    # half a step of bf16, relative
ULP32 = 2.0 ** -23    # a step of fp32: the most that one addition of the matrix unit is off by


def f64(bits):
    """bf16 bit patterns -> float64"""
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16(a):
    """float -> nearest bf16 value, as float64"""
    u = np.asarray(a, np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def mx_blocks(v):
    """v [R][K] -> (codes [R][ceil(K/32)][32] 0..15, exponents [R][ceil(K/32)], 128: NaN)"""
    R, K = v.shape
    nb = -(-K // 32)
    b = np.zeros((R, nb * 32))
    b[:, :K] = v
    b = b.reshape(R, nb, 32)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    X = np.where(top > 0, np.frexp(np.where(top > 0, top, 1.0))[1] - 3, -127)
    X = np.maximum(X, -127)
    a = np.abs(b) * np.exp2(-X.astype(np.float64))[..., None]
    d = np.abs(a[..., None] - E2M1)              # the nearest, the even code of two equally near
    near = d.min(-1, keepdims=True)
    cand = d == near
    even = cand & (np.arange(8) % 2 == 0)
    pick = np.where(even.any(-1), even.argmax(-1), cand.argmax(-1))
    codes = pick + 8 * np.signbit(b)
    return codes.astype(np.uint8), np.where(bad, 128, X).astype(np.int32)


def mx_values(v):
    codes, X = mx_blocks(v)
    a = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0) * np.exp2(X.astype(np.float64))[..., None]
    a = np.where((X == 128)[..., None], np.nan, a)
    return a.reshape(v.shape[0], -1)[:, :v.shape[1]]


def mx_packed(v):
    """(codes, scales) in the stored layout, zero bytes in the padding."""
    codes, X = mx_blocks(v)
    R, nb, _ = codes.shape
    R16, KT, KG = -(-R // 16), -(-v.shape[1] // 128), -(-v.shape[1] // 512)
    q = np.zeros((R16 * 16, KT * 4, 32), np.uint8)
    q[:R, :nb] = codes
    q = (q[..., 0::2] | (q[..., 1::2] << 4)).reshape(R16, 16, KT, 4, 16)
    s = np.zeros((R16 * 16, KG * 16), np.uint8)
    s[:R, :nb] = X + 127
    s = s.reshape(R16, 16, KG, 4, 4)             # tile, row, group, k tile of the group, block
    return q.transpose(0, 2, 3, 1, 4).reshape(R16, KT, 64, 16), s.transpose(0, 2, 4, 1, 3).reshape(R16, KG, 64, 4)


def lora(x, A, B, r):
    """((x A_r) B_r, bound of its fp32 evaluation with x A_r carried as two bf16 halves)"""
    out = np.zeros((x.shape[0], B.shape[2]))
    off = np.zeros_like(out)
    for c in range(A.shape[0]):
        i = np.nonzero(r == c)[0]
        if len(i) == 0:
            continue
        t, ta = x[i] @ A[c], np.abs(x[i]) @ np.abs(A[c])
        out[i] = t @ B[c]
        off[i] = ((x.shape[1] * ULP32 + HALF16 ** 2) * ta + 2 * A.shape[2] * ULP32 * np.abs(t)) @ np.abs(B[c])
    return out, off


def projection(x, W, A, B, r):
    """(x W + (x A_r) B_r, bound of its fp32 evaluation)"""
    h, off = x @ W, (x.shape[1] + 2) * ULP32 * (np.abs(x) @ np.abs(W))
    if A is not None:
        l, lo = lora(x, A, B, r)
        h, off = h + l, off + lo + ULP32 * np.abs(l)
    return h, off


def act(g, kind):
    """(act, act')"""
    erf = np.vectorize(math.erf)
    if kind == "gelu":
        p, slope = 0.5 * (1 + erf(g / math.sqrt(2))), np.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        p = np.where(g < -4, 0.5 * np.vectorize(math.erfc)(-g / math.sqrt(2)), p)
        return g * p, p + g * slope
    k = 2 * math.sqrt(2 / math.pi)
    y, dy = (g, 1.0) if kind == "silu" else (k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g))
    with np.errstate(over="ignore"):
        p, q = 1 / (1 + np.exp(-y)), 1 / (1 + np.exp(y))
    return g * p, p + g * p * q * dy


def gated(x, W, A, B, r, kind):
    h, _ = projection(x, W, A, B, r)
    F = h.shape[1] // 2
    return act(h[:, :F], kind)[0] * h[:, F:]


# |act'| <= 1.13 and |act''| <= 1 for all three; the fp32 evaluation of act and act' is off by the exponential's
# argument, (1 + |g|) steps and a handful more
SLOPE, CURVE = 1.13, 1.0


def gated_off(h, off, kind):
    F = h.shape[1] // 2
    g, u, eg, eu = h[:, :F], h[:, F:], off[:, :F], off[:, F:]
    a, _ = act(g, kind)
    return np.abs(u) * (SLOPE * eg + 8 * (2 + np.abs(g) ** 3) * ULP32 * np.abs(g)) + np.abs(a) * eu + SLOPE * eg * eu + HALF16 * np.abs(a * u)


def gated_gradients(dz, x, W, A, B, r, kind):
    """{name: (gradient, bound)}; dh is rounded to bf16 before the products, the results once more."""
    h, off = projection(x, W, A, B, r)
    F = h.shape[1] // 2
    g, u, eg, eu = h[:, :F], h[:, F:], off[:, :F], off[:, F:]
    a, da = act(g, kind)
    dh = np.concatenate((dz * u * da, dz * a), 1)
    own = 8 * (2 + np.abs(g) ** 3) * ULP32
    e = np.concatenate((np.abs(dz) * (np.abs(u) * (CURVE * eg + own) + (SLOPE + own) * eu), np.abs(dz) * (SLOPE * eg + own * np.abs(g))), 1)
    e = e + HALF16 * (np.abs(dh) + e)
    n = x.shape[0]
    out = {"dx": (dh @ W.T, (e + 2 * F * ULP32 * np.abs(dh)) @ np.abs(W).T),
           "dW": (x.T @ dh, np.abs(x).T @ (e + n * ULP32 * np.abs(dh)))}
    if A is not None:
        dx, ex = out["dx"]
        dA, eA, dB, eB = np.zeros_like(A), np.zeros_like(A), np.zeros_like(B), np.zeros_like(B)
        for c in range(A.shape[0]):
            i = np.nonzero(r == c)[0]
            s, t = dh[i] @ B[c].T, x[i] @ A[c]
            es = e[i] @ np.abs(B[c]).T + (2 * F * ULP32 + HALF16 ** 2) * (np.abs(dh[i]) @ np.abs(B[c]).T)
            et = (x.shape[1] * ULP32 + HALF16 ** 2) * (np.abs(x[i]) @ np.abs(A[c]))
            dx[i] += s @ A[c].T
            ex[i] += (es + 2 * A.shape[2] * ULP32 * np.abs(s)) @ np.abs(A[c]).T
            dA[c], eA[c] = x[i].T @ s, np.abs(x[i]).T @ (es + 2 * n * ULP32 * np.abs(s))
            dB[c], eB[c] = t.T @ dh[i], np.abs(t).T @ (e[i] + 2 * n * ULP32 * np.abs(dh[i])) + et.T @ (np.abs(dh[i]) + e[i])
        out |= {"dA": (dA, eA), "dB": (dB, eB)}
    return {k: (v, o + HALF16 * (np.abs(v) + o)) for k, (v, o) in out.items()}
