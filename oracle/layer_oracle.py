"""Plain fp64 definitions of the operators around the adapted expert
projections of an MoE layer: the input gradient through the experts, the
weighted sum of the expert outputs and its gradient, SwiGLU and its gradient,
and the 8-bit activation checkpoint.  Test infrastructure only; shares no code
with the library.

Arrays are numpy; P = T*k pairs p = t*k + j.  A pair is routed when its id is
in [0, E) and no lower slot of its token has the same id.
"""
import numpy as np


def routed(ids, E):
    """bool [T, k]"""
    ids = np.asarray(ids)
    ok = (ids >= 0) & (ids < E)
    for j in range(1, ids.shape[1]):
        for i in range(j):
            ok[:, j] &= ids[:, j] != ids[:, i]
    return ok


def expert_dx(dy, W, ids, E, absolute=False):
    """Per pair W_e^T dy[p], [P, d_in] (zero for dropped pairs).  absolute: the
    same sums of absolute values (the scale that rounding errors go by)."""
    ok = routed(ids, E).reshape(-1)
    flat = np.asarray(ids).reshape(-1)
    out = np.zeros((flat.size, W.shape[2]))
    for e in range(E):
        p = np.nonzero(ok & (flat == e))[0]
        if p.size:
            a, b = dy[p].astype(np.float64), W[e].astype(np.float64)
            out[p] = np.abs(a) @ np.abs(b) if absolute else a @ b
    return out


def slot_sum(rows, k):
    """[T*k, d] -> [T, d]"""
    return rows.reshape(-1, k, rows.shape[1]).sum(1)


def combine(y, w, ids, E):
    ok = routed(ids, E)
    T, k = ok.shape
    out = np.zeros((T, y.shape[1]))
    for t in range(T):
        for j in range(k):
            if ok[t, j]:
                out[t] += w[t, j] * y[t * k + j]
    return out


def combine_grads(dout, y, w, ids, E):
    """(dy [P, d], dw [T, k]), zero for dropped pairs."""
    ok = routed(ids, E)
    T, k = ok.shape
    dy, dw = np.zeros((T * k, dout.shape[1])), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            if ok[t, j]:
                dy[t * k + j] = w[t, j] * dout[t]
                dw[t, j] = np.dot(dout[t], y[t * k + j])
    return dy, dw


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def swiglu(g, u):
    return g * sigmoid(g) * u


def swiglu_grads(da, g, u):
    s = sigmoid(g)
    return da * u * s * (1.0 + g * (1.0 - s)), da * g * s


def pack(x):
    """(codes int8 [n, d], s uint8 [n, ceil(d/32)]) of fp32 or bf16 values given
    as fp64 (exactly)."""
    n, d = x.shape
    codes = np.zeros((n, d), np.int8)
    exps = np.zeros((n, -(-d // 32)), np.uint8)
    for b in range(exps.shape[1]):
        v = x[:, 32 * b:32 * b + 32]
        for i in range(n):
            top = np.max(np.abs(v[i]))
            if not np.isfinite(top):
                exps[i, b] = 255
                continue
            # exponent field of an fp32 number: 0 below 2^-126
            s = 0 if top < 2.0 ** -126 else int(np.floor(np.log2(top))) + 127
            if top >= 2.0 ** -126:      # log2 may be off by one next to a power of two
                while top >= 2.0 ** (s - 126):
                    s += 1
                while top < 2.0 ** (s - 127):
                    s -= 1
            if s < 254 and np.rint(top * 2.0 ** (133 - s)) >= 128:
                s += 1
            exps[i, b] = s
            codes[i, 32 * b:32 * b + 32] = np.clip(np.rint(v[i] * 2.0 ** (133 - s)), -127, 127)
    return codes, exps


def unpack(codes, exps):
    s = np.repeat(exps.astype(np.int64), 32, axis=1)[:, :codes.shape[1]]
    v = codes.astype(np.float64) * 2.0 ** (s - 133.0)
    return np.where(s == 255, np.nan, v)
