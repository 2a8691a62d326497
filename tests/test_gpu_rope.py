"""Rotary positions against the fp64 form (GPU).

Tolerance: one rounding to fp32 (2^-24 of the value) and the fp64 steps before
it, below 2^-40 of the pair's magnitudes at the positions used here (the
reference takes the same fp64 product pos * inv_freq)."""
import math

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


def check(y, x, pos, f, layout, mscale=1.0):
    want = ref.rotate(x, pos, f, layout, mscale)
    bound = 2.0 ** -24 * np.abs(want) + 2.0 ** -40 * np.abs(x).max() * abs(mscale)
    err = np.abs(y.astype(np.float64) - want)
    assert np.all(err <= bound), float((err / bound).max())
    n = 2 * len(f)
    assert np.array_equal(y[..., n:], x[..., n:])


@pytest.mark.parametrize("kind", ["none", "linear", "parts"])
@pytest.mark.parametrize("n,base", [(2, 10000.0), (64, 10000.0), (122, 500000.0), (1024, 1e6)])
def test_frequencies(kind, n, base):
    f = w4.rope_frequencies(n, base, kind, 8.0, 4096).cpu().numpy()
    want = ref.frequencies(n, base, kind, 8.0, 4096)
    assert np.all(np.abs(f - want) <= 2.0 ** -48 * want)


def test_frequencies_by_parts_with_equal_ends():
    f = w4.rope_frequencies(8, 10000.0, "parts", 4.0, 64, beta_fast=1.0, beta_slow=1.0)
    want = ref.frequencies(8, 10000.0, "parts", 4.0, 64, 1.0, 1.0)
    assert np.allclose(f.cpu().numpy(), want, rtol=1e-14)


# one token and a few, rows by rows and several to a workgroup, whole heads and
# parts of them, pairs that fall on 16-byte units and pairs that do not
@pytest.mark.parametrize("T,NH,D,n", [
    (1, 1, 4, 2), (1, 16, 256, 64), (3, 5, 128, 122), (7, 2, 64, 64), (33, 3, 96, 50),
    (5, 64, 128, 128), (1100, 1, 64, 16), (2100, 2, 32, 6), (600, 16, 128, 128), (2, 1, 1024, 1024)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation(T, NH, D, n, layout):
    g = synth.rng(T + n)
    x = synth.normal_f32(g, (T, NH, D))
    pos = g.integers(-100, 200000, T).astype(np.int32)
    f = ref.frequencies(n, 10000.0)
    y = w4.rope_rotate(dev(x), dev(pos), dev(f), layout)
    check(y.cpu().numpy(), x, pos, f, layout)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n", [64, 54])
def test_rotation_in_place_strided_and_scaled(layout, n):
    """A slice of a fused projection's rows, in place and into another slice;
    what lies around the slices stays."""
    T, NH, D = 9, 4, 64
    g = synth.rng(5)
    buf = synth.normal_f32(g, (T, 8, D))
    pos = (np.arange(T) * 40000 - 7).astype(np.int32)
    f = ref.frequencies(n, 500000.0, "parts", 8.0, 4096)
    ms = float(np.float32(1 + 0.1 * math.log(8)))
    b = dev(buf)
    out = torch.full((T, 6, D), 7.0, device="cuda")
    w4.rope_rotate(b[:, 2:6], dev(pos), dev(f), layout, ms, out=out[:, 1:5])
    check(out[:, 1:5].cpu().numpy(), buf[:, 2:6], pos, f, layout, ms)
    assert bool((out[:, 0] == 7.0).all()) and bool((out[:, 5] == 7.0).all())
    w4.rope_rotate(b[:, 2:6], dev(pos), dev(f), layout, ms, out=b[:, 2:6])
    assert torch.equal(b[:, 2:6], out[:, 1:5])
    assert np.array_equal(b[:, :2].cpu().numpy(), buf[:, :2])
    assert np.array_equal(b[:, 6:].cpu().numpy(), buf[:, 6:])


def test_far_positions_keep_their_angles():
    """Positions near 2^31: the angle is still good to 2^-20 of a turn (fp64
    holds it to 2^-53 of 2^31 radians), where fp32 would have lost it."""
    pos = np.array([2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7], np.int32)
    x = np.zeros((3, 1, 4), np.float32)
    x[:, 0, 0] = 1.0
    f = np.array([1.0, 0.1])
    y = w4.rope_rotate(dev(x), dev(pos), dev(f)).cpu().numpy()
    for t, p in enumerate(pos.tolist()):
        assert abs(y[t, 0, 0] - math.cos(p)) < 1e-6 and abs(y[t, 0, 2] - math.sin(p)) < 1e-6


def test_infinities_and_nan_stay_in_their_pairs():
    x = np.ones((1, 1, 8), np.float32)
    x[0, 0, 1], x[0, 0, 2] = np.inf, np.nan
    y = w4.rope_rotate(dev(x), dev(np.array([3], np.int32)), dev(ref.frequencies(8))).cpu().numpy()[0, 0]
    assert np.isfinite(y[[0, 4, 3, 7]]).all() and not np.isfinite(y[[1, 5, 2, 6]]).any()


def test_empty_call():
    x = torch.empty(0, 4, 64, device="cuda")
    p = torch.empty(0, dtype=torch.int32, device="cuda")
    assert w4.rope_rotate(x, p, w4.rope_frequencies(64)).shape == (0, 4, 64)
