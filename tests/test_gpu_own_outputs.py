"""Outputs that a call makes itself, on a stream that is not the current one
(GPU): they must not be memory that the current stream's pending work still
writes."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def attention_calls():
    g = synth.rng(1)
    c = attn_cases.random_plan(g, [200, 64], [9, 5], 2, 128, "q4_0")
    kv = attn_cases.on_gpu(c)
    r = lambda *s: torch.randn(*s, device="cuda")
    q, k, v, x = r(14, 8, 128), r(14, 2, 128), r(14, 2, 128), r(6, 5000)
    f, pos = w4.rope_frequencies(64), torch.arange(14, dtype=torch.int32, device="cuda")
    t = torch.arange(6, dtype=torch.int32, device="cuda")
    return {
        "rope_frequencies": lambda s: [w4.rope_frequencies(128, stream=s)],
        "rope_rotate": lambda s: [w4.rope_rotate(q, pos, f, stream=s)],
        "kv_append": lambda s: [w4.kv_append(kv, k, v, pos=pos, inv_freq=f, q=q, stream=s)],
        "kv_read": lambda s: list(w4.kv_read(kv, 14, stream=s)),
        "attn_forward": lambda s: list(w4.attn_forward(kv, q, 0.1, stream=s)),
        "token_logprobs": lambda s: list(w4.token_logprobs(x, t, 4, stream=s)),
    }


def check(call):
    want = [t.clone() for t in call(None)]
    st = torch.cuda.Stream()
    busy = torch.ones(4096, 4096, device="cuda")
    call(st)
    torch.cuda.synchronize()
    for _ in range(3):
        # two of each, freed with a write to them still queued on the current stream
        old = [torch.empty_like(t) for t in want for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(100):
            busy = torch.tanh(busy)
        for t in old:
            t.fill_(7)
        del t, old
        got = call(st)
        st.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del got, a, b


@pytest.mark.parametrize("name", ["rope_frequencies", "rope_rotate", "kv_append", "kv_read", "attn_forward",
                                  "token_logprobs"])
def test_attention_side_calls(name):
    check(attention_calls()[name])
