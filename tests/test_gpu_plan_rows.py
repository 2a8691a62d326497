"""Calls with fewer rows than the plan's sequences have (GPU): row r of
sequence s is token kv_len[s] - (cu_rows[s+1] - r) all the same."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases, attn_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


# the last row of the call inside a sequence, at its end, before others
@pytest.mark.parametrize("T", [1, 3, 5, 6, 30, 39])
@pytest.mark.parametrize("D,fmt", [(64, "q4_0"), (128, "q4_sym")])
def test_the_first_rows_of_a_plan(T, D, fmt):
    g = synth.rng(T + D)
    c = attn_cases.random_plan(g, [70, 3, 300], [5, 5, 30], 2, D, fmt)     # (two rows before token 0)
    kv = attn_cases.on_gpu(c)
    k, v, q = (synth.normal_f32(g, (c.T, h, D)) for h in (2, 2, 8))
    before = [t.clone() for t in kv.tensors[:2]]
    w4.kv_append(kv, dev(k), dev(v))
    whole = [t.clone() for t in kv.tensors[:2]]
    ko, vo = w4.kv_read(kv, c.T)
    a, b = w4.kv_read(kv, T)
    assert torch.equal(a, ko[:T]) and torch.equal(b, vo[:T])
    # attention of the first T rows
    out, lse = w4.attn_forward(kv, dev(q[:T]), 0.1)
    c.k_pool, c.v_pool = (t.cpu().numpy() for t in whole)
    r = ref.attention(c, q, 0.1)
    bo, bl = ref.attention_bounds(r)
    l = lse.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(out.cpu().numpy() - r.out[:T]) <= bo[:T])
    seen = np.isfinite(r.lse[:T])
    assert np.array_equal(np.isfinite(l), seen)
    assert np.all(np.abs(l - r.lse[:T])[seen] <= bl[:T][seen])
    # the first T rows stored, then all of them: the first T's bytes were in their places
    for t, x in zip(kv.tensors, before):
        t.copy_(x)
    w4.kv_append(kv, dev(k[:T]), dev(v[:T]))
    a, b = w4.kv_read(kv, c.T)
    assert torch.equal(a[:T], ko[:T]) and torch.equal(b[:T], vo[:T])
    for t, x, y in zip(kv.tensors, before, whole):
        assert bool(((t == x) | (t == y)).all())


def test_a_window_with_the_first_rows():
    g = synth.rng(5)
    c = attn_cases.random_plan(g, [400], [200], 1, 64, "q4_0")
    q = 2.0 * synth.normal_f32(g, (200, 4, 64))
    r = ref.attention(c, q, 0.125, 70)
    bo, _ = ref.attention_bounds(r)
    for T in (1, 50, 199):
        out, _ = w4.attn_forward(attn_cases.on_gpu(c), dev(q[:T]), 0.125, 70)
        assert np.all(np.abs(out.cpu().numpy() - r.out[:T]) <= bo[:T]), T
