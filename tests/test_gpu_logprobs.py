"""Token log probabilities, entropy and top alternatives against fp64 (GPU).
Tolerances: attn_ref.logprobs counts the roundings; ids are exact."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def check(x, targets, n, got, what=""):
    lp, ent, ids, top, blp, bent, btop = ref.logprobs(x, targets, n)
    f = lambda t: t.cpu().numpy().astype(np.float64)

    def near(a, b, bound, name):
        # a difference of two fp32 numbers can lie past fp32's range
        b = np.where(np.abs(b) > np.finfo(np.float32).max, np.copysign(np.inf, b), b)
        fin = np.isfinite(b)
        assert np.array_equal(np.isnan(a), np.isnan(b)), (what, name)
        assert np.array_equal(a[~fin & ~np.isnan(b)], b[~fin & ~np.isnan(b)]), (what, name)
        e = np.abs(a[fin] - b[fin])
        assert np.all(e <= bound[fin] + 1e-44), (what, name, float((e / (bound[fin] + 1e-44)).max()))

    if targets is not None:
        near(f(got[0]), lp, blp, "logprob")
    near(f(got[1]), ent, bent, "entropy")
    if n:
        assert np.array_equal(got[2].cpu().numpy(), ids), (what, "ids")
        near(f(got[3]), top, btop, "top")


# one value, around the 4-value groups, a wave's chunk (1024) and a workgroup's
# (4096), several spans of one row and one span a row
@pytest.mark.parametrize("V", [1, 2, 5, 63, 1023, 1024, 1027, 4096, 4099, 32001, 151936])
@pytest.mark.parametrize("T,n", [(1, 20), (3, 1), (2, 0)])
def test_logprobs(T, V, n):
    n = min(n, V)
    g = synth.rng(V + T)
    x = synth.normal_f32(g, (T, V), 3.0)
    t = g.integers(0, V, T).astype(np.int32)
    t[0] = int(x[0].argmax())
    check(x, t, n, w4.token_logprobs(dev(x), dev(t), n))


@pytest.mark.parametrize("T,V,n", [(600, 1500, 32), (520, 4099, 3), (40, 20011, 32)])
def test_many_rows(T, V, n):
    g = synth.rng(T)
    x = synth.normal_f32(g, (T, V), 2.0)
    x[np.arange(T), g.integers(0, V, T)] += (30 * g.random(T)).astype(np.float32)   # confident rows
    t = g.integers(0, V, T).astype(np.int32)
    check(x, t, n, w4.token_logprobs(dev(x), dev(t), n))


@pytest.mark.parametrize("off", [0, 1, 2, 3])
def test_strided_rows(off):
    """Rows that start at every offset from a 16-byte boundary, with
    infinities and NaN between them."""
    T, V = 5, 2049
    g = synth.rng(off)
    buf = np.full((T, V + 4 + off), np.nan, np.float32)
    buf[:, V:V + 2] = np.inf
    buf[:, :V] = synth.normal_f32(g, (T, V))
    t = np.array([0, V - 1, 5, -1, V], np.int32)
    got = w4.token_logprobs(dev(buf)[:, :V], dev(t), 7)
    check(buf[:, :V], t, 7, got)
    assert float(got[0][3]) == 0.0 and float(got[0][4]) == 0.0


def rows(V):
    """Rows in which the selection or the sums can go wrong."""
    g = synth.rng(V)
    up = np.arange(V, dtype=np.float32)
    few = np.full(V, -np.inf, np.float32)
    few[[3, V // 2, V - 1]] = [1.0, 2.0, 1.0]
    one = np.full(V, -np.inf, np.float32)
    one[V - 2] = -5.0
    lowest = np.full(V, -np.finfo(np.float32).max)
    mixed = lowest.copy()
    mixed[7] = 4.0
    wide = np.where(np.arange(V) % 2, 3e38, -3e38).astype(np.float32)
    conf = synth.normal_f32(g, (V,))
    conf[11] = 40.0
    zeros = np.zeros(V, np.float32)
    zeros[1::2] = -0.0
    ties = np.round(synth.normal_f32(g, (V,))).astype(np.float32)
    tiny = np.full(V, -1e30, np.float32)
    tiny[5] = -1e30 + 1e25
    return {"ascending": up, "descending": up[::-1].copy(), "equal": np.full(V, 2.5, np.float32),
            "zeros": zeros, "ties": ties, "few": few, "one": one, "none": np.full(V, -np.inf, np.float32),
            "lowest": lowest, "lowest and one": mixed, "wide": wide, "confident": conf,
            "far below zero": tiny}


@pytest.mark.parametrize("V", [37, 1500, 9001])
@pytest.mark.parametrize("n", [1, 32])
def test_hard_rows(V, n):
    for name, r in rows(V).items():
        x = np.stack([r, r])
        t = np.array([V - 2, int(np.argmax(r))], np.int32)
        check(x, t, n, w4.token_logprobs(dev(x), dev(t), n), name)
    # the same rows, one span each
    names, x = zip(*rows(V).items())
    x = np.concatenate([np.stack(x)] * 40)
    t = np.full(len(x), 3, np.int32)
    check(x, t, n, w4.token_logprobs(dev(x), dev(t), n), "together")


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_rows_with_nan_or_infinity(bad):
    V, n = 5000, 5
    g = synth.rng(9)
    x = synth.normal_f32(g, (3, V))
    x[1, 4321] = bad
    x[1, 17] = bad
    x[2, :] = bad
    t = np.array([1, 2, 3], np.int32)
    check(x, t, n, w4.token_logprobs(dev(x), dev(t), n))


def test_one_workspace_for_calls_of_several_shapes():
    """Its arrival counters are zero after each call."""
    g = synth.rng(13)
    shapes = [(1, 151936, 20), (3, 9000, 32), (400, 9001, 1), (7, 50, 5), (2, 70000, 0)]
    ws = torch.zeros(max(w4.logprobs_workspace(*s).numel() for s in shapes), dtype=torch.uint8, device="cuda")
    for T, V, n in shapes + shapes[::-1]:
        x, t = synth.normal_f32(g, (T, V), 3.0), g.integers(0, V, T).astype(np.int32)
        check(x, t, n, w4.token_logprobs(dev(x), dev(t), n, workspace=ws), (T, V, n))
        assert not bool(ws[:2048].any())


def test_parts_of_the_result():
    """Each output on its own gives the same bits; nothing else is needed."""
    g = synth.rng(12)
    x, t = dev(synth.normal_f32(g, (3, 9000))), dev(np.array([1, 2, 3], np.int32))
    a = w4.token_logprobs(x, t, 4)
    b = w4.token_logprobs(x, t, want_entropy=False)
    c = w4.token_logprobs(x, None, 4, want_entropy=False)
    assert b[1] is None and b[2] is None and c[0] is None
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], c[2]) and torch.equal(a[3], c[3])
    assert w4.token_logprobs(x[:0], t[:0], 4)[2].shape == (0, 4)


@pytest.mark.parametrize("V", [7, 40000])
def test_a_confident_rows_small_log_probability(V):
    """Two values, the rest -infinity: log p of the larger is -log1p(exp(-d)),
    to 2^-21 relative.  d is exact; exp's first-order term takes log(2) as fp32,
    2^-28 |d| off (2^-22.4 at 45), exp2 is off by 2^-23, the correction's, the
    sums' and log1p's roundings by 2^-24, 2^-24 and 2^-23: 6.5 2^-24 in all."""
    d = np.array([0.5, 3.3, 7.9, 13.1, 19.7, 23.7, 31.3, 44.9], np.float32)
    x = np.full((len(d), V), -np.inf, np.float32)
    x[:, V - 2] = 1.0
    x[np.arange(len(d)), np.arange(len(d)) % (V - 3)] = np.float32(1.0) - d
    gap = 1.0 - x[np.arange(len(d)), np.arange(len(d)) % (V - 3)].astype(np.float64)
    want = -np.log1p(np.exp(-gap))
    got = w4.token_logprobs(dev(x), dev(np.full(len(d), V - 2, np.int32)))[0].cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want) <= 2.0 ** -21 * np.abs(want)), (got, want)
