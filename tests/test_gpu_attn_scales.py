"""Attention over value scales that lie far apart (GPU): what a key that a row
does not see, or gives next to no probability, holds does not enter the row.
Tolerances: attn_seen.attention, made of the keys that the row sees."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases, attn_ref as ref, attn_seen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def case(seed, lens, rows, NH, NKV, D, fmt):
    g = synth.rng(seed)
    c = attn_cases.random_plan(g, lens, rows, NKV, D, fmt)
    return c, 2.0 * synth.normal_f32(g, (c.T, NH, D))


def scales(pool, c, s, tok, h):
    """The NB scales of token `tok` of sequence s as a view."""
    nb = c.D // 32
    sc = pool[c.table[s, tok // 64], h, nb * 1024:].view(np.float16 if c.fmt == "q4_0" else np.float32)
    t = tok % 64
    return sc.reshape(nb, 64)[:, t % 16 // 4 * 16 + t // 16 * 4 + t % 4]


def compare(got, want, rows=slice(None)):
    o, l, bo, bl = want
    eo = np.abs(got[0].cpu().numpy().astype(np.float64) - o)[rows] / bo[rows]
    el = np.abs(got[1].cpu().numpy().astype(np.float64) - l)[rows] / bl[rows]
    assert np.all(eo <= 1.0) and np.all(el <= 1.0), (float(np.nanmax(eo)), float(np.nanmax(el)))


# rows and heads of every tile: 4, 8, 16 and 32 rows, waves that share a block
# and waves of two; two or four tiles see the last token
SHAPES = [([130], [2], 2, 1, 64), ([300], [4], 2, 1, 256), ([300], [4], 4, 2, 128), ([200], [64], 16, 1, 64),
          ([270], [17], 256, 1, 256), ([700], [520], 64, 1, 128), ([200], [190], 256, 1, 64),
          ([90], [70], 512, 1, 256)]


@pytest.mark.parametrize("fmt,low,high", [("q4_0", 2.0 ** -10, 6e4), ("q4_sym", 1.0, 1e8), ("q4_sym", 1.0, 2.0 ** 40),
                                          ("q4_sym", 2.0 ** -40, 2.0 ** 100), ("q4_sym", 2.0 ** 100, 2.0 ** 40)])
@pytest.mark.parametrize("lens,rows,NH,NKV,D", SHAPES)
def test_a_scale_that_only_the_last_token_sees(lens, rows, NH, NKV, D, fmt, low, high):
    c, q = case(sum(lens) + D, lens, rows, NH, NKV, D, fmt)
    for p in range(c.v_pool.shape[0]):
        for h in range(NKV):
            sc = c.v_pool[p, h, D // 32 * 1024:].view(np.float16 if fmt == "q4_0" else np.float32)
            sc[:] = (sc.astype(np.float64) * low).astype(sc.dtype)
    want = attn_seen.attention(c, q, 0.125)
    for h in range(NKV):
        scales(c.v_pool, c, 0, lens[0] - 1, h)[::2] = high      # and not in every block
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125)
    compare(got, want, slice(0, c.T - 1))
    compare([t[-1:] for t in got], [a[-1:] for a in attn_seen.attention(c, q, 0.125)])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [150, 3000])
@pytest.mark.parametrize("away,high", [(20.0, 1e8), (60.0, 2.0 ** 60), (80.0, 2.0 ** 100)])
def test_a_scale_of_a_key_without_probability(D, n, away, high):
    """Keys that the row sees, with a score so far below the others that they
    count for little whatever their size."""
    NKV, scale = 2, 0.125
    c, q = case(n + D, [n], [1], NKV, NKV, D, "q4_sym")
    for tok in (3, n // 2, n - 1):
        for h in range(NKV):
            page, nb = c.table[0, tok // 64], D // 32
            codes = ref.tile_rows(c.k_pool[page, h], D, "q4_sym", True)[0][tok % 64].astype(np.float64) - 8
            dots = (codes * ref.values8(q[0, h:h + 1], "q4_sym").reshape(nb, 32)).sum(1)
            scales(c.k_pool, c, 0, tok, h)[:] = -np.sign(dots) * away / (scale * np.abs(dots).sum())
            scales(c.v_pool, c, 0, tok, h)[:] = high
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), scale)
    compare(got, attn_seen.attention(c, q, scale))


@pytest.mark.parametrize("step", [0.3, -0.3, 1.5])
@pytest.mark.parametrize("n,rows,NH,D,window", [(700, 40, 2, 64, 0), (700, 3, 2, 256, 0), (160, 100, 16, 128, 30)])
def test_scales_that_grow_and_fall_along_the_sequence(n, rows, NH, D, window, step):
    """By 2^step a token, up to 2^100 apart: rows of a tile see other largest
    scales, and other least ones."""
    c, q = case(n + D, [n], [rows], NH, 1, D, "q4_sym")
    for tok in range(n):
        sc = scales(c.v_pool, c, 0, tok, 0)
        sc[:] = sc * np.float32(2.0 ** np.clip(step * (tok - n + 66), -100, 100))
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125, window)
    compare(got, attn_seen.attention(c, q, 0.125, window))


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
def test_scales_far_apart_in_runs_that_are_joined(fmt):
    for D, lens, rows, NH in ((128, [9000], [1], 8), (256, [6000], [2], 4), (64, [5000, 40, 900], [1, 3, 2], 2)):
        c, q = case(D, lens, rows, NH, 1, D, fmt)
        for s, n in enumerate(lens):
            for tok in range(5, n, 17):
                sc = scales(c.v_pool, c, s, tok, 0)
                sc[:] = (sc.astype(np.float64) * 2.0 ** (-12 if tok % 2 else 14 if fmt == "q4_0" else 30)).astype(sc.dtype)
        got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125)
        compare(got, attn_seen.attention(c, q, 0.125))


def test_infinite_and_nan_scales_beside_far_ones():
    """Where a step's scales lie far apart too, a NaN or infinite scale reaches
    the rows that see it only, and its own columns."""
    D, NH = 64, 2
    c, q = case(6, [130], [6], NH, 1, D, "q4_sym")
    scales(c.v_pool, c, 0, 40, 0)[:] *= np.float32(1e-12)
    scales(c.v_pool, c, 0, 129, 0)[:] = 1e12
    want = attn_seen.attention(c, q, 0.125)
    for tok, x in ((128, np.nan), (127, np.inf)):
        scales(c.v_pool, c, 0, tok, 0)[0] = x
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125)
    compare(got, want, slice(0, 3))
    o = got[0].cpu().numpy()
    assert not np.isfinite(o[3:, :, :32]).any()
    bo = want[2][3:, :, 32:]
    assert np.all(np.abs(o[3:, :, 32:] - want[0][3:, :, 32:]) <= bo)
