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


def older_calls():
    g = synth.rng(2)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda")
    r = lambda *s: d(synth.normal_f32(g, s))
    M, N, K = 9, 512, 256
    x, w, wq, ws = r(M, K), r(N, K), d(synth.q4_0_random_blocks(g, N, K)), d(synth.q4_sym_random_blocks(g, N, K))
    xq, x1, xs = w4.q8_0_quantize(x), w4.q8_0_quantize(x[0]), w4.q8_f32_quantize(x[0])
    T, H, I, E, k = 4, 512, 256, 8, 2
    hid, y, gamma, rl = r(T, H), r(T, H), r(H), r(T, E)
    ids, wts = (d(a) for a in synth.routing(g, T, E, k))
    q4 = [d(synth.q4_0_random_blocks(g, n, m)) for n, m in ((E * 2 * I, H), (E * H, I), (2 * I, H), (H, I))]
    sym = [d(synth.q4_sym_random_blocks(g, n, m)) for n, m in ((E * 2 * I, H), (E * H, I), (2 * I, H), (H, I))]
    mws, sws = w4.moe_workspace(T, H, I, E, k), w4.moe_sym_workspace(T, H, I, E, k)
    gdn = [d(a) for a in synth.gdn_inputs(g, 40, 2, 128, 128)[:5]]
    return {
        "q8_0_quantize": lambda s: [w4.q8_0_quantize(x, stream=s)],
        "q4_0_quantize": lambda s: [w4.q4_0_quantize(w, stream=s)],
        "q4_sym_quantize": lambda s: [w4.q4_sym_quantize(w, stream=s)],
        "q8_f32_quantize": lambda s: [w4.q8_f32_quantize(x, stream=s)],
        "q4q8_gemv": lambda s: [w4.q4q8_gemv(wq, x1, N, K, stream=s)],
        "q4sym_q8f32_gemv": lambda s: [w4.q4sym_q8f32_gemv(ws, xs, N, K, stream=s)],
        "q4q8_gemm": lambda s: [w4.q4q8_gemm(wq, xq, M, N, K, stream=s)],
        "gdn_scan": lambda s: list(w4.gdn_scan(*gdn, stream=s)),
        "router_topk": lambda s: list(w4.router_topk(rl, k, stream=s)),
        "rmsnorm_residual": lambda s: list(w4.rmsnorm_residual(hid, y, gamma, stream=s)),
        "moe_workspace": lambda s: [w4.moe_workspace(T, H, I, E, k, stream=s)],
        "moe_forward": lambda s: [w4.moe_forward(hid, ids, wts, *q4, H, I, E, k, mws, stream=s)],
        "moe_forward_noalloc": lambda s: [w4.moe_forward_noalloc(hid, ids, wts, *q4, H, I, E, k, stream=s)],
        "moe_layer": lambda s: list(w4.moe_layer(hid, y, gamma, ids, wts, *q4, H, I, E, k, mws, stream=s)),
        "moe_layer_routed": lambda s: list(w4.moe_layer_routed(hid, y, gamma, rl, *q4, H, I, E, k, mws, stream=s)),
        "moe_sym_forward": lambda s: [w4.moe_sym_forward(hid, ids, wts, *sym, H, I, E, k, sws, stream=s)],
    }


@pytest.mark.parametrize("name", ["q8_0_quantize", "q4_0_quantize", "q4_sym_quantize", "q8_f32_quantize", "q4q8_gemv",
                                  "q4sym_q8f32_gemv", "q4q8_gemm", "gdn_scan", "router_topk", "rmsnorm_residual",
                                  "moe_workspace", "moe_forward", "moe_forward_noalloc", "moe_layer",
                                  "moe_layer_routed", "moe_sym_forward"])
def test_layer_and_product_calls(name):
    check(older_calls()[name])
