"""Plans whose cu_rows decrease (GPU): attention writes nothing and leaves its
workspace ready for the next call."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("D,NH,room", [(64, 4, None), (128, 8, None), (256, 8, 1000)])    # joined in the launch, or by another
@pytest.mark.parametrize("falling", [[0, 40, 0, 40], [0, 40, 0, 7], [40, 0, 40, 39], [3, 50, 41, 41], [-5, 8, -9, 40],
                                     [0, 0, 40, 39]])
def test_rows_that_decrease(falling, D, NH, room):
    g = synth.rng(D)
    c = attn_cases.random_plan(g, [3000, 700, 5000], [20, 1, 19], 2, D, "q4_0", capacity=room)
    kv = attn_cases.on_gpu(c)
    q = torch.from_numpy(2.0 * synth.normal_f32(g, (40, NH, D))).to("cuda")
    ws = w4.attn_workspace(kv, 40, NH)
    want = w4.attn_forward(kv, q, 0.1, workspace=ws)
    good = kv.tensors[4].clone()
    kv.tensors[4].copy_(torch.tensor(falling, dtype=torch.int32))
    out, lse = torch.full_like(want[0], 7.0), torch.full_like(want[1], 7.0)
    w4.attn_forward(kv, q, 0.1, out=out, lse=lse, workspace=ws)
    assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
    assert not bool(ws[:12288].any())
    kv.tensors[4].copy_(good)
    got = w4.attn_forward(kv, q, 0.1, workspace=ws)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_many_sequences_of_which_one_decreases():
    g = synth.rng(2)
    B = 200
    c = attn_cases.random_plan(g, [90] * B, [1] * B, 1, 64, "q4_0")
    kv = attn_cases.on_gpu(c)
    q = torch.from_numpy(synth.normal_f32(g, (B, 2, 64))).to("cuda")
    for at in (1, 64, 128, 199):
        cu = c.cu.copy()
        cu[at] = cu[at + 1] + 1
        kv.tensors[4].copy_(torch.from_numpy(cu))
        out = torch.full((B, 2, 64), 7.0, device="cuda")
        w4.attn_forward(kv, q, 0.125, out=out)
        assert bool((out == 7.0).all()), at
