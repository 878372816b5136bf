"""The gated block's definition and the bounds of its roundings (block_reference.py) in 64 bits on the device, for
sizes that take long in numpy.  The same formulas; the activations by way of erfc and exp alone."""
import math

import torch

import block_reference as ref

HALF16, ULP32 = ref.HALF16, ref.ULP32


def mm(a, b):
    return torch.matmul(a.contiguous(), b.contiguous())


def lora(x, A, B, r):
    out = torch.zeros(x.shape[0], B.shape[2], dtype=torch.float64, device=x.device)
    off = torch.zeros_like(out)
    for c in range(A.shape[0]):
        i = torch.nonzero(r == c).flatten()
        if len(i):
            t, ta = mm(x[i], A[c]), mm(x[i].abs(), A[c].abs())
            out[i] = mm(t, B[c])
            off[i] = mm((x.shape[1] * ULP32 + HALF16 ** 2) * ta + 2 * A.shape[2] * ULP32 * t.abs(), B[c].abs())
    return out, off


def projection(x, W, A, B, r):
    h, off = mm(x, W), (x.shape[1] + 2) * ULP32 * mm(x.abs(), W.abs())
    if A is not None:
        l, lo = lora(x, A, B, r)
        h, off = h + l, off + lo + ULP32 * l.abs()
    return h, off


def act(g, kind):
    """(act, act')"""
    if kind == "gelu":
        p, slope = 0.5 * torch.special.erfc(-g / math.sqrt(2)), torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        return g * p, p + g * slope
    k = 2 * math.sqrt(2 / math.pi)
    y, dy = (g, 1.0) if kind == "silu" else (k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g))
    p, q = 1 / (1 + torch.exp(-y)), 1 / (1 + torch.exp(y))
    return g * p, p + g * p * q * dy


def gated_off(h, off, kind):
    F = h.shape[1] // 2
    g, u, eg, eu = h[:, :F], h[:, F:], off[:, :F], off[:, F:]
    a, _ = act(g, kind)
    own = 8 * (2 + g.abs() ** 3) * ULP32 * g.abs()
    return u.abs() * (ref.SLOPE * eg + own) + a.abs() * eu + ref.SLOPE * eg * eu + HALF16 * (a * u).abs()


def gradients(dz, x, W, A, B, r, kind):
    h, off = projection(x, W, A, B, r)
    F, n = h.shape[1] // 2, x.shape[0]
    g, u, eg, eu = h[:, :F], h[:, F:], off[:, :F], off[:, F:]
    a, da = act(g, kind)
    dh = torch.cat((dz * u * da, dz * a), 1)
    own = 8 * (2 + g.abs() ** 3) * ULP32
    e = torch.cat((dz.abs() * (u.abs() * (ref.CURVE * eg + own) + (ref.SLOPE + own) * eu), dz.abs() * (ref.SLOPE * eg + own * g.abs())), 1)
    e = e + HALF16 * (dh.abs() + e)
    out = {"dx": [mm(dh, W.t()), mm(e + 2 * F * ULP32 * dh.abs(), W.abs().t())],
           "dW": [mm(x.t(), dh), mm(x.abs().t(), e + n * ULP32 * dh.abs())]}
    if A is not None:
        dA, eA, dB, eB = torch.zeros_like(A), torch.zeros_like(A), torch.zeros_like(B), torch.zeros_like(B)
        for c in range(A.shape[0]):
            i = torch.nonzero(r == c).flatten()
            if len(i) == 0:
                continue
            xi, di, ei, Bt, rank = x[i], dh[i], e[i], B[c].t().contiguous(), A.shape[2]
            s, t = mm(di, Bt), mm(xi, A[c])
            es = mm(ei, Bt.abs()) + (2 * F * ULP32 + HALF16 ** 2) * mm(di.abs(), Bt.abs())
            et = (x.shape[1] * ULP32 + HALF16 ** 2) * mm(xi.abs(), A[c].abs())
            out["dx"][0][i] += mm(s, A[c].t())
            out["dx"][1][i] += mm(es + 2 * rank * ULP32 * s.abs(), A[c].abs().t())
            dA[c], eA[c] = mm(xi.t(), s), mm(xi.abs().t(), es + 2 * n * ULP32 * s.abs())
            dB[c], eB[c] = mm(t.t(), di), mm(t.abs().t(), ei + 2 * n * ULP32 * di.abs()) + mm(et.t(), di.abs() + ei)
        out |= {"dA": [dA, eA], "dB": [dB, eB]}
    return {k: (v, o + HALF16 * (v.abs() + o)) for k, (v, o) in out.items()}
