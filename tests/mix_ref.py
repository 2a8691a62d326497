"""Plain forms (numpy, fp64) of the 8-bit rows and their product, the short
convolution and the state space scan, each with the bound of its fp32 error.

U = 2^-24 is half a step of fp32 relative to the value: what one rounding may
be off.  The bounds count roundings, times the sum of the magnitudes of what
is added."""
import numpy as np

U = 2.0 ** -24
PAD = 128


def quantize(x):
    """Codes int8 [rows, KP] and scales fp32 [rows], every step one binary32
    operation."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    with np.errstate(all="ignore"):
        d = (np.abs(x).max(1) * (np.float32(1) / np.float32(127))).astype(np.float32)
        inv = np.where(d == 0, np.float32(0), np.float32(1) / d).astype(np.float32)
        inv[np.isinf(inv)] = 0
        v = (x * inv[:, None]).astype(np.float32).astype(np.float64)
        c = np.clip(np.trunc(v + np.copysign(0.5, v)), -127, 127)
    bad = ~np.isfinite(x).all(1)
    d[bad], c[bad] = np.nan, 0
    q = np.zeros((M, -(-K // PAD) * PAD), np.int8)
    q[:, :K] = c.astype(np.int8)
    return q, d


def product(xq, xd, wq, wd, bias=None):
    """The product in 64 bits and its bound: the sum's conversion, the scales'
    product, the two together and the bias are one rounding each."""
    s = xq.astype(np.float64) @ wq.astype(np.float64).T
    y = s * (xd.astype(np.float64)[:, None] * wd.astype(np.float64)[None])
    bound = 3 * U * np.abs(y) * (1 + 1e-6)
    if bias is not None:
        y = y + bias.astype(np.float64)
    return y, bound + U * np.abs(y) * (1 + 1e-6)


def silu(v):
    return v / (1.0 + np.exp(-v))


def silu_bound(v, e):
    """SiLU of an argument that is off by e: |SiLU'| <= 1.1; then the base-2
    exponent's product and constant (2 U |v| of e^-v), exp2 and the reciprocal
    (an ulp, 2 U, each), the sum and the product; results below fp32's normal
    range may be 0."""
    return 1.1 * e + (6 + 2 * np.abs(v)) * U * np.abs(silu(v)) * (1 + 1e-6) + 1e-36


def conv(cu, src, dst, x, w, bias, state, act):
    """Outputs of the rows of sequences (others NaN), the bound, new states."""
    W, CH = w.shape
    T = len(x)
    y, b = np.full((T, CH), np.nan), np.zeros((T, CH))
    new = None if state is None else state.copy()
    w64 = w.astype(np.float64)
    for s in range(len(cu) - 1):
        r0, r1 = min(max(cu[s], 0), T), min(max(cu[s + 1], 0), T)
        if r1 <= r0:
            continue
        old = state[src[s]] if state is not None and 0 <= src[s] < len(state) else np.zeros((W - 1, CH))
        ext = np.concatenate([old, x[r0:r1]]).astype(np.float64)
        n = r1 - r0
        v = sum(ext[i:i + n] * w64[i] for i in range(W))
        mag = sum(np.abs(ext[i:i + n] * w64[i]) for i in range(W))
        if bias is not None:
            v, mag = v + bias, mag + np.abs(bias)
        e = (W + 1) * U * mag * (1 + 1e-6)         # W products with sums, the bias
        y[r0:r1], b[r0:r1] = (silu(v), silu_bound(v, e)) if act == "silu" else (v, e)
        if state is not None and 0 <= dst[s] < len(state):
            new[dst[s]] = ext[n:].astype(np.float32)
    return y, b, new


def scan(cu, src, dst, x, dt, A, B, C, state, D=None, z=None, dt_bias=None, softplus=True):
    """Outputs of the rows of sequences (others NaN), new states, and the
    bounds of both.

    What may be off in an entry of S: U times 4 roundings a row of everything
    it is made of (R: the row's product with its step, the decay, the sum, and
    those of a chunk's product), 16 roundings of each term (its step: softplus;
    its weight: two exponentials and products), and of each term the exponent
    of its decay, which is off by the steps' and the exponent's own roundings,
    12 U relative (Z: the terms weighted by their exponents).  An output sums N
    such entries and 64 products within the chunk, each once rounded, and few
    roundings more (D, the joins)."""
    T, NH, P = x.shape
    NG, N = B.shape[1:]
    G = NH // NG
    y, by = np.full((T, NH, P), np.nan), np.zeros((T, NH, P))
    new = None if state is None else state.astype(np.float64)
    bnew = None if state is None else np.zeros(state.shape)
    f = lambda a: a.astype(np.float64)
    for s in range(len(cu) - 1):
        r0, r1 = min(max(cu[s], 0), T), min(max(cu[s + 1], 0), T)
        if r1 <= r0:
            continue
        S = f(state[src[s]]) if state is not None and 0 <= src[s] < len(state) else np.zeros((NH, N, P))
        M = np.abs(S)
        R, Z = np.zeros_like(M), np.zeros_like(M)
        for t in range(r0, r1):
            # (dt + dt_bias is rounded once before what follows)
            v = f(dt[t]) if dt_bias is None else f((dt[t] + dt_bias).astype(np.float32))
            d = np.logaddexp(0, v) if softplus else v
            lg = (d * f(A))[:, None, None]
            keep = np.exp(lg)
            bt, ct = np.repeat(f(B[t]), G, 0), np.repeat(f(C[t]), G, 0)
            new_term = bt[:, :, None] * (d[:, None] * f(x[t]))[:, None, :]
            S = keep * S + new_term
            Z = keep * (Z + np.abs(lg) * M)
            M = keep * M + np.abs(new_term)
            R = keep * R + M
            o = np.einsum("hn,hnp->hp", ct, S)
            e = U * (4 * R + 16 * M + 12 * Z)
            mag = np.einsum("hn,hnp->hp", np.abs(ct), M)
            eo = np.einsum("hn,hnp->hp", np.abs(ct), e) + U * (N + 64 + 8) * mag
            if D is not None:
                o = o + f(D)[:, None] * f(x[t])
                eo = eo + 3 * U * np.abs(f(D)[:, None] * f(x[t]))
            if z is not None:
                g = f(z[t])
                eo = eo * np.abs(silu(g)) + np.abs(o) * silu_bound(g, 0) + U * np.abs(o * silu(g))
                o = o * silu(g)
            y[t], by[t] = o, eo
        if state is not None and 0 <= dst[s] < len(state):
            new[dst[s]], bnew[dst[s]] = S, U * (4 * R + 16 * M + 12 * Z)
    return y, by + 1e-36, new, None if bnew is None else bnew + 1e-36
