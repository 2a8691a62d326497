"""fp64 attention with bounds made of the keys that a row sees alone."""
import numpy as np

from tests import attn_ref as ref


def attention(c, q, scale, window=0):
    """Of plan c (see attn_ref.attention, all pages present): out and lse, and
    per element the error allowed:
      - (2 ds + 2^-20 + n 2^-23) sum p |v| as in attn_ref.attention_bounds;
      - a product p d (p = 1 for the largest score) of a probability and a
        value scale goes in as two fp16 halves.  Where the scales met lie within
        2^13 of each other the largest of them stands at 2^14 .. 2^15, the least
        at 2^2 or more, and fp16's smallest step is 2^-24: 2^-25 is 2^-27 of the
        least scale.  Otherwise the row's own largest product stands at 2^14 or
        more: 2^-25 is 2^-39 of it.  Times a code of up to 8, a key."""
    T, NH, D = q.shape
    G, nb = NH // c.k_pool.shape[1], D // 32
    xq = ref.values8(q, c.fmt)
    out, lse = np.zeros((T, NH, D)), np.full((T, NH), -np.inf)
    bo, bl = np.full((T, NH, D), 1e-37), np.full((T, NH), 2.0 ** -22)
    for s in range(len(c.len)):
        n, r0, r1 = int(c.len[s]), int(c.cu[s]), int(c.cu[s + 1])
        pages = c.table[s, :-(-n // ref.PAGE)]
        for h in range(c.k_pool.shape[1]):
            def rows(pool, is_k):
                t = [ref.tile_rows(pool[p, h], D, c.fmt, is_k) for p in pages]
                return (np.concatenate([a for a, _ in t])[:n].astype(np.float64) - 8,
                        np.concatenate([b for _, b in t])[:n].astype(np.float64))
            kc, kd = rows(c.k_pool, True)
            vc, vd = rows(c.v_pool, False)
            for row in range(r0, r1):
                i = n - (r1 - row)
                see = slice(max(0, i - window + 1) if window else 0, max(0, i + 1))
                if see.start >= see.stop:
                    continue
                d = np.abs(vd[see])                                      # [keys, blocks]
                V = (vc[see] * vd[see][..., None]).reshape(len(d), D)
                o = slice(h * G, (h + 1) * G)
                x = xq[row, o].reshape(G, nb, 32)
                terms = np.stack([x[:, b] @ (kc[see, b] * kd[see, b, None]).T for b in range(nb)], -1) * scale
                sc = terms.sum(2)                                        # [heads, keys]
                m = sc.max(1)
                p = np.exp(sc - m[:, None])
                z = p.sum(1)
                out[row, o], lse[row, o] = (p / z[:, None]) @ V, m + np.log(z)
                ds = 2.0 ** -24 * ((nb + 2) * np.abs(terms).sum(2).max(1) + 8 * np.abs(sc).max(1) + 4)
                adds = len(d) / 16 + 80
                least = np.where(d > 0, d, np.inf).min(0)
                least = np.where(np.isfinite(least), least, 0.0)
                most = np.stack([(p * d[:, b]).max(1) for b in range(nb)], 1)
                tail = len(d) * (2.0 ** -24 * least + 2.0 ** -36 * most)
                rel = 2 * ds + 2.0 ** -20 + adds * 2.0 ** -23
                bo[row, o] += rel[:, None] * ((p / z[:, None]) @ np.abs(V)) + np.repeat(tail, 32, 1)
                bl[row, o] += ds + adds * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse[row, o])
    return out, lse, bo, bl
