"""Top alternatives of rows in which many tokens share the largest logits:
uniform, clipped or coarsely quantized logits over an allowed set (GPU).  Ids
are exact; log probabilities within attn_ref.logprobs' count of roundings."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def check(rows, n, copies):
    """`rows` [R, V], each `copies` times in one call."""
    x = torch.from_numpy(rows).to("cuda").repeat(copies, 1)
    _, _, ids, top = w4.token_logprobs(x, None, n, want_entropy=False)
    _, _, want, wtop, *_, bound = ref.logprobs(rows, None, n)
    got = ids.cpu().numpy().reshape(copies, len(rows), n)
    wrong = (got != want).any((0, 2))
    assert not wrong.any(), (np.flatnonzero(wrong).tolist(), got[0][wrong][0].tolist(), want[wrong][0].tolist())
    err = np.abs(top.cpu().numpy().astype(np.float64).reshape(got.shape) - wtop)
    assert np.all(err <= bound), float((err / bound).max())


def tied(V, part, level=10.0):
    """Four rows, `part` of whose tokens stand at `level`, above all others."""
    g = synth.rng(int(V + 1000 * part))
    x = np.minimum(synth.normal_f32(g, (4, V)), np.float32(6.0))
    x[g.random((4, V)) < part] = level
    return x


# one span a row, where the rows fill the card, and several
@pytest.mark.parametrize("copies", [1, 130])
@pytest.mark.parametrize("n", [1, 5, 20, 32])
@pytest.mark.parametrize("part", [0.005, 0.01, 0.02, 0.05])
@pytest.mark.parametrize("V", [32000, 151936])
def test_sparse_ties_at_the_maximum(V, part, n, copies):
    check(tied(V, part), n, copies)


@pytest.mark.parametrize("copies", [1, 130])
@pytest.mark.parametrize("n", [5, 32])
def test_ties_below_the_largest_and_coarse_logits(n, copies):
    V = 151936
    g = synth.rng(n)
    x = tied(V, 0.01)
    x[0, [V - 1, 7]] = 11.0, 12.0                        # a few larger ones
    x[1] = -np.inf                                       # an allowed set, all alike
    x[1, g.random(V) < 0.02] = -3.0
    x[2] = np.round(2.0 * synth.normal_f32(g, (V,))) / 4
    x[3] = np.where(g.random(V) < 0.03, np.float32(0.0), np.float32(-0.0)) - \
        np.where(g.random(V) < 0.9, np.float32(1.0), np.float32(0.0))      # 0 and -0 are equal
    check(x, n, copies)


@pytest.mark.parametrize("n", [1, 32])
@pytest.mark.parametrize("part", [0.01, 0.05])
def test_ties_of_a_row_in_many_spans(part, n):
    """More than 64 spans a row, so that four waves join them."""
    check(tied(1 << 20, part)[:1], n, 1)


def test_ties_at_infinity_and_nan():
    """Sparse +infinity, and sparse NaN: their ids, by index, and NaN."""
    V, n = 151936, 20
    for bad in (np.inf, np.nan):
        x = tied(V, 0.02, bad)
        _, _, ids, top = w4.token_logprobs(torch.from_numpy(x).to("cuda"), None, n)
        assert np.array_equal(ids.cpu().numpy(), ref.logprobs(x, None, n)[2])
        assert bool(torch.isnan(top).all())
