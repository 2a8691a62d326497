"""Attention with scores far from zero (GPU)."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases, attn_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
@pytest.mark.parametrize("D,lens,rows,NH,NKV", [
    (64, [300], [1], 2, 1), (128, [150, 40], [20, 9], 4, 2), (256, [90], [90], 16, 1), (64, [600], [520], 64, 1),
    (128, [9000], [1], 8, 1)])
@pytest.mark.parametrize("size", [1e5, 3e6, 1e7, 1e8, 3e9, 1e15, 1e35])
def test_large_scores(size, D, lens, rows, NH, NKV, fmt):
    """Scores of about `size`.  The log sum is as accurate as a score is.  A row
    whose two largest scores lie further apart than twice their error and 40
    more has the largest's value: to the 2^-20 of a product of two halves and
    the final division, and of each other key exp(-40) and the halves' least
    step, 2^-27 of a scale times a code of up to 8.  Any row stays among the
    values that it sees, a weighted mean whose weights and sums are rounded."""
    g = synth.rng(D + lens[0])
    c = attn_cases.random_plan(g, lens, rows, NKV, D, fmt)
    q = 2.0 * synth.normal_f32(g, (c.T, NH, D))
    scale = size / (2.0 * 1.3 * D ** 0.5)           # rows of q and K of norm 2 sqrt(D) and about 1.3 sqrt(D)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    out, lse = w4.attn_forward(attn_cases.on_gpu(c), dev(q), scale)
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    scale = float(np.float32(scale))
    nb, G, xq, sure, all_ = D // 32, NH // NKV, ref.values8(q, fmt), 0, 0
    for s in range(len(lens)):
        pages = c.table[s, :-(-lens[s] // 64)]
        for h in range(NKV):
            def rows_of(pool, is_k):
                t = [ref.tile_rows(pool[p, h], D, fmt, is_k) for p in pages]
                return np.concatenate([(a.astype(np.float64) - 8) * b.astype(np.float64)[..., None]
                                       for a, b in t])[:lens[s]].reshape(-1, D)
            K, V = rows_of(c.k_pool, True), rows_of(c.v_pool, False)
            for row in range(c.cu[s], c.cu[s + 1]):
                n = lens[s] - (int(c.cu[s + 1]) - row) + 1
                for o in {h * G, (h + 1) * G - 1}:
                    all_ += 1
                    terms = (K[:n] * xq[row, o]).reshape(n, nb, 32).sum(2) * scale
                    sc = terms.sum(1)
                    ds = 2.0 ** -24 * ((nb + 2) * np.abs(terms).sum(1).max() + 8 * np.abs(sc).max() + 4)
                    order = np.argsort(sc)
                    best = order[-1]
                    assert abs(lse[row, o] - sc[best]) <= ds + np.log(n) + 2.0 ** -22 * abs(sc[best])
                    lo, hi, big = V[:n].min(0), V[:n].max(0), np.abs(V[:n]).max()
                    assert np.all(out[row, o] >= lo - 2.0 ** -12 * big) and np.all(out[row, o] <= hi + 2.0 ** -12 * big)
                    if n == 1 or sc[best] - sc[order[-2]] > 2 * ds + 40:
                        sure += 1
                        assert np.all(np.abs(out[row, o] - V[best]) <= 2.0 ** -20 * np.abs(V[best]) +
                                      n * (2.0 ** -24 + np.exp(-40.0)) * big)
    assert sure >= all_ // 2
