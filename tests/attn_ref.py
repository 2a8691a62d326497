"""Plain fp64 forms of rotary positions, the paged 4-bit cache, attention over
it and token log probabilities, for the tests (numpy; the block formats from
the oracle).  Shares no code with the HIP sources."""
from __future__ import annotations

import math

import numpy as np

import oracle

PAGE = 64


# ------------------------------------------------------------------ rotary positions
def frequencies(n, base=10000.0, kind="none", factor=1.0, orig_len=0, fast=32.0, slow=1.0):
    f = np.array([base ** (-2.0 * i / n) for i in range(n // 2)])
    if kind == "linear":
        return f / factor
    if kind == "parts":
        pair = lambda turns: n * math.log(orig_len / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(pair(fast))), min(n - 1, math.ceil(pair(slow)))
        mix = np.clip((np.arange(n // 2) - lo) / max(hi - lo, 0.001), 0, 1)
        return f * (1 - mix) + f / factor * mix
    return f


def rotate(x, pos, f, layout="half", mscale=1.0):
    """x [T, NH, D] turned, in fp64."""
    n = 2 * len(f)
    y = np.array(x, np.float64)
    a = np.asarray(pos, np.float64)[:, None, None] * f
    c, s = np.cos(a) * mscale, np.sin(a) * mscale
    ia, ib = (np.arange(n // 2), np.arange(n // 2) + n // 2) if layout == "half" else \
        (np.arange(0, n, 2), np.arange(1, n, 2))
    xa, xb = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia] = xa * c - xb * s
    y[..., ib] = xb * c + xa * s
    return y


# ------------------------------------------------------------------ blocks
# Q4_0 comes from the oracle.  The others take a scale as the binary32 product
# with the rounded reciprocal of 7 or 127; apart from the scale their steps are
# the oracle's Q4_SYM, Q8_0 and Q8_F32, which test_attn_abi.py checks.
def _away(v):
    t = np.trunc(v)
    return np.where(np.abs(v - t) >= 0.5, t + np.sign(v), t)


def _scaled(x, n):
    b = np.ascontiguousarray(x, np.float32).reshape(-1, x.shape[-1] // 32, 32)
    return b, np.abs(b).max(-1) * (np.float32(1.0) / np.float32(n))


def _codes(b, d, n):
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        inv = np.float32(1.0) / d
    inv = np.where((d == 0) | np.isinf(inv), np.float32(0), inv)
    return np.clip(_away(b * inv[..., None]), -n, n)


def codes4(x, fmt):
    """4-bit rows: (codes 0..15 with the value (code - 8) * d, scales)."""
    if fmt == "q4_sym":
        b, d = _scaled(x, 7)
        return (_codes(b, d, 7) + 8).astype(np.uint8), d
    rows = np.ascontiguousarray(x, np.float32).reshape(-1, x.shape[-1])
    b = np.asarray(oracle.q4_0_quantize(rows)).reshape(rows.shape[0], -1, 18)
    d = np.ascontiguousarray(b[..., :2]).view(np.float16)[..., 0]
    return np.concatenate([b[..., 2:] & 15, b[..., 2:] >> 4], -1), d


def values8(x, fmt):
    """8-bit rows: the values they stand for, fp64."""
    b, d = _scaled(x, 127)
    if fmt == "q4_0":
        d = d.astype(np.float16).astype(np.float32)
    return (_codes(b, d, 127).astype(np.float64) * d.astype(np.float64)[..., None]).reshape(x.shape)


# ------------------------------------------------------------------ page tiles
def tile_bytes(D, fmt):
    return D // 32 * (1024 + PAGE * (2 if fmt == "q4_0" else 4))


def put(pool, page, h, t, codes, d, fmt, is_k):
    """Row t of a tile: codes [NB, 32] and scales [NB] written as the header
    lays them out."""
    nb = codes.shape[0]
    tile = pool[page, h]
    sc = tile[nb * 1024:].view(np.float16 if fmt == "q4_0" else np.float32)
    for b in range(nb):
        for j in range(16):
            lo, hi = int(codes[b, j]), int(codes[b, j + 16])
            if is_k:
                c, i = divmod(j, 4)
                at = 4 * (b * 256 + c * 64 + (t % 16) * 4 + t // 16) + i
                tile[at] = (lo ^ 8) | (hi ^ 8) << 4
            else:
                at = b * 1024 + (t % 16) // 4 * 256 + j * 16 + t // 16 * 4 + (0, 2, 1, 3)[t % 4]
                tile[at] = lo | hi << 4
        sc[b * 64 + (t % 16) // 4 * 16 + t // 16 * 4 + t % 4] = d[b]


def _maps(nb):
    t, j = np.arange(PAGE)[:, None], np.arange(16)[None, :]
    k = 4 * ((j // 4) * 64 + (t % 16) * 4 + t // 16) + j % 4
    v = (t % 16) // 4 * 256 + j * 16 + t // 16 * 4 + np.array([0, 2, 1, 3])[t % 4]
    s = (t % 16) // 4 * 16 + t // 16 * 4 + t % 4
    return k, v, s[:, 0]


def tile_rows(tile, D, fmt, is_k):
    """All 64 rows of a tile: (codes 0..15 [64, NB, 32], scales [64, NB])."""
    nb = D // 32
    km, vm, sm = _maps(nb)
    raw = tile[:nb * 1024].reshape(nb, 1024)
    by = raw[:, km if is_k else vm].transpose(1, 0, 2)
    codes = np.concatenate([by & 15, by >> 4], -1)
    if is_k:
        codes = codes ^ 8
    sc = tile[nb * 1024:].view(np.float16 if fmt == "q4_0" else np.float32).reshape(nb, PAGE)
    return codes, sc[:, sm].T


# ------------------------------------------------------------------ attention
class Result:
    pass


def attention(c, q, scale, window=0):
    """fp64 attention of q [T, NH, D] on the plan c (k_pool, v_pool, table, len,
    cu, D, fmt), with the magnitudes tolerances are made of: r.mag = sum p |v|
    per element and r.ds, the largest error of a score from fp32 rounding."""
    T, NH, D = q.shape
    n_pages, NKV = c.k_pool.shape[:2]
    G, nb = NH // NKV, D // 32
    xq = values8(q, c.fmt)
    r = Result()
    r.out, r.mag = np.zeros((T, NH, D)), np.zeros((T, NH, D))
    r.lse, r.ds = np.full((T, NH), -np.inf), np.zeros((T, NH))
    r.keys = np.zeros(T, np.int64)
    r.dmax = np.zeros((T, NH))       # largest finite value scale of the sequence's tokens
    for s in range(len(c.len)):
        r0, r1 = int(c.cu[s]), int(c.cu[s + 1])
        n = min(int(c.len[s]), c.table.shape[1] * PAGE)
        if r1 <= r0 or n <= 0:
            continue
        pages = c.table[s, :-(-n // PAGE)]
        ok = (pages >= 0) & (pages < n_pages)
        there = np.repeat(ok, PAGE)[:n]
        for h in range(NKV):
            def rows(pool, is_k):
                got = []
                for p, o in zip(pages, ok):
                    if o:
                        codes, d = tile_rows(pool[p, h], D, c.fmt, is_k)
                    else:
                        codes, d = np.full((PAGE, nb, 32), 8, np.uint8), np.zeros((PAGE, nb))
                    got.append((codes.astype(np.float64) - 8) * d.astype(np.float64)[..., None])
                return np.concatenate(got)[:n].reshape(n, D)
            with np.errstate(invalid="ignore"):
                K, V = rows(c.k_pool, True), rows(c.v_pool, False)
            dv = np.concatenate([tile_rows(c.v_pool[p, h], D, c.fmt, False)[1] if o else np.zeros((PAGE, nb))
                                 for p, o in zip(pages, ok)])[:n]
            r.dmax[r0:r1, h * G:(h + 1) * G] = np.abs(dv[np.isfinite(dv)]).max(initial=0.0)
            for row in range(r0, r1):
                i = int(c.len[s]) - (r1 - row)
                j = np.arange(n)
                see = (j <= i) & there
                if window:
                    see &= j > i - window
                r.keys[row] = see.sum()
                if not see.any():
                    continue
                Kr, Vr = K[see], V[see]
                for g in range(G):
                    x = xq[row, h * G + g]
                    terms = (Kr * x).reshape(-1, nb, 32).sum(2) * scale
                    sc = terms.sum(1)
                    m = sc.max()
                    e = np.exp(sc - m)
                    z = e.sum()
                    o = h * G + g
                    r.out[row, o] = (e / z) @ Vr
                    r.mag[row, o] = (e / z) @ np.abs(Vr)
                    r.lse[row, o] = m + math.log(z)
                    # nb + 2 roundings of partial sums no larger than sum |terms|; the factor's own
                    # rounding and the product's against the maximum, a few units of |s|; exp2's own
                    a = np.abs(terms).sum(1).max()
                    r.ds[row, o] = 2.0 ** -24 * ((nb + 2) * a + 8 * np.abs(sc).max() + 4)
    return r


def attention_bounds(r):
    """(bound on |out|'s error, bound on lse's).  A probability is off by ds
    relative to the others twice over (its own and the sum's); each product
    enters with 21 bits (two fp16 halves, the lower one rounded), of which the
    last is no finer than half of 2^-24, fp16's smallest step, where the largest
    value scale stands at 2^14 or more: 2^-25 * dmax / 2^14 times a code of up to
    8 is 2^-36 dmax a key, over a sum of probabilities of at least 1; sums of n
    fp32 additions: one for 16 keys of a wave's page, the pages' in turn, then
    four waves and up to 16 and 32 partial results."""
    n = r.keys[:, None] / 16 + 80
    rel = 2 * r.ds + 2.0 ** -20 + n * 2.0 ** -23
    with np.errstate(invalid="ignore"):
        lse = r.ds + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(np.isfinite(r.lse), r.lse, 0.0))
    tail = r.keys[:, None] * 2.0 ** -36 * r.dmax
    return rel[..., None] * r.mag + tail[..., None] + 1e-37, lse + 2.0 ** -22


# ------------------------------------------------------------------ log probabilities
def logprobs(x, targets, n):
    """(logprob, entropy, ids, top, bounds of the first two and the last)."""
    x = np.asarray(x, np.float64)
    T, V = x.shape
    lp, ent = np.zeros(T), np.zeros(T)
    blp, bent = np.zeros(T), np.zeros(T)
    ids, top, btop = np.zeros((T, n), np.int32), np.zeros((T, n)), np.zeros((T, n))
    # additions in a row: a chunk of 16, the chunks of a lane, lanes, waves, spans
    adds = 16 + V / 64 / 4 / 16 + 6 + 4 + 64
    for t in range(T):
        r = x[t]
        key = np.where(np.isnan(r), np.inf, r)
        order = np.lexsort((np.arange(V), -key, ~np.isnan(r)))[:n]
        ids[t] = order
        g = None if targets is None else int(targets[t])
        if np.isnan(r).any() or np.isposinf(r).any():
            lp[t] = 0.0 if g is not None and not 0 <= g < V else np.nan
            ent[t] = np.nan
            top[t] = np.nan
            continue
        if np.isneginf(r).all():
            lp[t] = 0.0 if g is not None and not 0 <= g < V else -np.inf
            top[t] = -np.inf
            continue
        at = int(r.argmax())
        d = r - r[at]
        e = np.exp(d)
        e[at] = 0.0
        z = e.sum()
        lz = math.log1p(z)
        dd = np.where(e > 0, d, 0.0)
        ent[t] = lz - (e * dd).sum() / (1 + z)
        # a term: its difference's rounding and the base-2 product's, 2^-23 (1 + |d|) relative, and exp2's
        te = e * 2.0 ** -22 * (1 + np.abs(dd))
        bz = (te.sum() + z * adds * 2.0 ** -24) / (1 + z)
        blz = bz + 2.0 ** -22 * lz
        bent[t] = blz + 2.0 ** -23 * ent[t] + ((te * np.abs(dd)).sum() + (e * np.abs(dd)).sum() *
                                               (adds + 4) * 2.0 ** -24) / (1 + z) * 1.01
        if g is not None and 0 <= g < V:
            lp[t] = d[g] - lz
            blp[t] = blz + 2.0 ** -23 * (abs(d[g]) + lz) if np.isfinite(d[g]) else 0.0
        top[t] = d[order] - lz
        btop[t] = np.where(np.isfinite(top[t]), blz + 2.0 ** -23 * (np.abs(d[order]) + lz), 0.0)
    return lp, ent, ids, top, blp, bent, btop
