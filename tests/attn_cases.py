"""Synthetic paged 4-bit caches for the GPU tests (numpy, seeded)."""
import types

import numpy as np

from tests import attn_ref as ref


def random_plan(g, lens, rows, NKV, D, fmt, spare=2, capacity=None, scale=1.0):
    """Sequences of `lens` tokens, the last `rows` of each this call's, on pages
    in any order of the pool; random codes, scales near those of N(0, scale^2)
    rows.  Scales and codes of tokens past a sequence's end are NaN and any."""
    per = [-(-n // ref.PAGE) for n in lens]
    P = sum(per) + spare
    cap = capacity or max(per + [1]) + 1
    nb, n = D // 32, ref.tile_bytes(D, fmt)
    ft = np.float16 if fmt == "q4_0" else np.float32

    def pool():
        x = g.integers(0, 256, (P, NKV, n)).astype(np.uint8)
        d = (g.uniform(0.22, 0.36, (P, NKV, nb * 64)) * g.choice([-1, 1], (P, NKV, nb * 64)) * scale).astype(ft)
        x[..., nb * 1024:] = d.view(np.uint8).reshape(P, NKV, -1)
        return x

    c = types.SimpleNamespace(k_pool=pool(), v_pool=pool(), D=D, fmt=fmt)
    order = g.permutation(P)
    c.table = np.full((len(lens), cap), -1, np.int32)
    at = 0
    for s, k in enumerate(per):
        c.table[s, :k] = order[at:at + k]
        at += k
        if lens[s] % 64:      # the rest of the last page: never written
            for pl in (c.k_pool, c.v_pool):
                sc = pl[order[at - 1]][:, nb * 1024:].view(ft)
                for b in range(nb):
                    for t in range(lens[s] % 64, 64):
                        sc[:, b * 64 + (t % 16) // 4 * 16 + t // 16 * 4 + t % 4] = np.nan
    c.len = np.array(lens, np.int32)
    c.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    c.T = int(c.cu[-1])
    return c


def on_gpu(c):
    import torch

    import paper_2606_24031_amd as w4
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    return w4.KVCache(dev(c.k_pool), dev(c.v_pool), dev(c.table), dev(c.len), dev(c.cu), c.D, c.fmt)
