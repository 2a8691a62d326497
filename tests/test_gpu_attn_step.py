"""Rotary positions, the cache, attention and the log probabilities run
together as a served model's token step does, eagerly, from a captured graph
and on a stream of its own (GPU)."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases, attn_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

NH, NKV, D, V = 8, 2, 128, 2048


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


class Session:
    """Two requests: a prompt each, then one token a step."""

    def __init__(self, seed, lens=(150, 40), room=4, fmt="q4_0"):
        self.g = synth.rng(seed)
        self.B, self.lens, self.fmt = len(lens), np.array(lens), fmt
        self.kp, self.vp = w4.kv_pools(self.B * room, NKV, D, fmt)
        self.kp.fill_(0xFF)                       # NaN scales everywhere
        self.vp.fill_(0xFF)
        order = self.g.permutation(self.B * room).reshape(self.B, room).astype(np.int32)
        self.table = dev(order)
        self.f = w4.rope_frequencies(64, 10000.0)
        self.K = [np.zeros((0, NKV, D), np.float32) for _ in lens]
        self.V = [np.zeros((0, NKV, D), np.float32) for _ in lens]

    def step(self, rows):
        """One call's projections and plan for `rows` tokens of each request,
        which become their last."""
        T = sum(rows)
        self.qkv = synth.normal_f32(self.g, (T, NH + 2 * NKV, D))
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.pos = np.concatenate([np.arange(n - r, n) for n, r in zip(self.lens, rows)]).astype(np.int32)
        k = ref.rotate(self.qkv[:, NH:NH + NKV], self.pos, ref.frequencies(64)).astype(np.float32)
        for s in range(self.B):
            a = slice(self.cu[s], self.cu[s + 1])
            self.K[s] = np.concatenate([self.K[s], k[a]])
            self.V[s] = np.concatenate([self.V[s], self.qkv[a, NH + NKV:]])

    def want(self):
        """fp64 from the rows themselves: (out, bound on its error)."""
        q = ref.rotate(self.qkv[:, :NH], self.pos, ref.frequencies(64)).astype(np.float32)
        xq = ref.values8(q, self.fmt)
        val = lambda x: ((lambda c, d: (c.astype(np.float64) - 8) * d.astype(np.float64)[..., None])
                         (*ref.codes4(x, self.fmt))).reshape(x.shape)
        out, mag = np.zeros(q.shape), np.zeros(q.shape)
        for s in range(self.B):
            K, Vv = val(self.K[s]), val(self.V[s])
            for r in range(self.cu[s], self.cu[s + 1]):
                for h in range(NH):
                    n = self.pos[r] + 1
                    sc = K[:n, h // (NH // NKV)] @ xq[r, h] * D ** -0.5
                    p = np.exp(sc - sc.max())
                    p /= p.sum()
                    out[r, h], mag[r, h] = p @ Vv[:n, h // (NH // NKV)], p @ np.abs(Vv[:n, h // (NH // NKV)])
        return out, 2.0 ** -16 * mag + 1e-9      # of attn_ref.attention_bounds, at |s| < 16 and 200 keys

    def plan(self):
        return w4.KVCache(self.kp, self.vp, self.table, dev(self.lens.astype(np.int32)), dev(self.cu), D, self.fmt)


def forward(kv, qkv, pos, f, head, targets):
    q = w4.kv_append(kv, qkv[:, NH:NH + NKV], qkv[:, NH + NKV:], pos=pos, inv_freq=f, q=qkv[:, :NH])
    o, lse = w4.attn_forward(kv, q, D ** -0.5)
    xq = w4.q8_0_quantize(o.reshape(o.shape[0], -1))
    logits = w4.q4q8_gemm(head, xq, o.shape[0], V, NH * D)
    return [q, o, lse, logits, *w4.token_logprobs(logits, targets, 4)]


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
def test_prompt_and_steps(fmt):
    s = Session(1, fmt=fmt)
    head = dev(synth.q4_0_random_blocks(s.g, V, NH * D))
    for i in range(4):
        rows = list(s.lens) if i == 0 else [1, 1]
        if i:
            s.lens = s.lens + 1
        s.step(rows)
        t = s.g.integers(0, V, sum(rows)).astype(np.int32)
        q, o, lse, logits, lp, ent, ids, top = forward(s.plan(), dev(s.qkv), dev(s.pos), s.f, head, dev(t))
        want, bound = s.want()
        assert np.all(np.abs(o.cpu().numpy() - want) <= bound), i
        x = logits.cpu().numpy()
        rlp, rent, rids, rtop, blp, bent, btop = ref.logprobs(x, t, 4)
        assert np.array_equal(ids.cpu().numpy(), rids)
        assert np.all(np.abs(lp.cpu().numpy() - rlp) <= blp) and np.all(np.abs(ent.cpu().numpy() - rent) <= bent)


def test_a_captured_step_replayed_as_the_requests_grow():
    """The step captured once; between replays the inputs, kv_len and the
    positions change in place and other eager calls run on the device."""
    s = Session(2, lens=(62, 1))
    head = dev(synth.q4_0_random_blocks(s.g, V, NH * D))
    s.step(list(s.lens))
    forward(s.plan(), dev(s.qkv), dev(s.pos), s.f, head, dev(np.zeros(63, np.int32)))
    s.lens = s.lens + 1
    s.step([1, 1])
    kv = s.plan()
    qkv, pos, t = dev(s.qkv), dev(s.pos), dev(np.array([5, 6], np.int32))
    want = forward(kv, qkv, pos, s.f, head, t)          # warms up; the same rows are stored again below
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = forward(kv, qkv, pos, s.f, head, t)
    for i in range(5):
        if i:
            s.lens = s.lens + 1
            s.step([1, 1])
            qkv.copy_(dev(s.qkv))
            pos.copy_(dev(s.pos))
            kv.tensors[3].copy_(dev(s.lens.astype(np.int32)))
        for x in got:
            x.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        o = got[1].cpu().numpy()
        ref_o, bound = s.want()
        assert np.all(np.abs(o - ref_o) <= bound), i
        eager = forward(kv, qkv, pos, s.f, head, t)
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b), i
        if i == 0:
            for a, b in zip(want, eager):
                assert torch.equal(a, b)


def test_on_another_stream():
    """Every call on a stream that is not the current one, given by `stream`,
    and as the current one."""
    s = Session(3)
    s.step(list(s.lens))
    kv = s.plan()
    b, pos = dev(s.qkv), dev(s.pos)
    st = torch.cuda.Stream()
    T = int(s.cu[-1])
    x = torch.randn(T, 3000, device="cuda")
    torch.cuda.synchronize()
    q = w4.kv_append(kv, b[:, NH:NH + NKV], b[:, NH + NKV:], pos=pos, inv_freq=s.f, q=b[:, :NH], stream=st)
    ws = w4.attn_workspace(kv, T, NH, stream=st)
    o, lse = w4.attn_forward(kv, q, D ** -0.5, workspace=ws, stream=st)
    lw = w4.logprobs_workspace(T, 3000, 3, stream=st)
    r = w4.token_logprobs(x, None, 3, workspace=lw, stream=st)
    st.synchronize()
    want, bound = s.want()
    assert np.all(np.abs(o.cpu().numpy() - want) <= bound)
    with torch.cuda.stream(st):
        r2 = w4.token_logprobs(x, None, 3)
    st.synchronize()
    assert torch.equal(r[2], r2[2]) and torch.equal(r[3], r2[3])


def test_two_calls_at_once_with_their_own_workspaces():
    """Two streams, two plans over one pool, at the same time: each gives what
    it gives alone."""
    g = synth.rng(6)
    cs = [attn_cases.random_plan(g, [9000, 30], [1, 2], 2, 128, "q4_0") for _ in range(2)]
    qs = [dev(2 * synth.normal_f32(g, (3, 8, 128))) for _ in cs]
    kvs = [attn_cases.on_gpu(c) for c in cs]
    alone = [w4.attn_forward(kv, q, 0.09) for kv, q in zip(kvs, qs)]
    ws = [w4.attn_workspace(kv, 3, 8) for kv in kvs]
    out = [torch.empty(3, 8, 128, device="cuda") for _ in cs]
    lse = [torch.empty(3, 8, device="cuda") for _ in cs]
    st = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            w4.attn_forward(kvs[i], qs[i], 0.09, out=out[i], lse=lse[i], workspace=ws[i], stream=st[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(out[i], alone[i][0]) and torch.equal(lse[i], alone[i][1])


def test_graphs_that_share_a_workspace():
    """Graphs of calls of several shapes (runs joined within the launch, by a
    second one, not split) on one workspace, replayed in turn with eager calls
    on it between; log probabilities on theirs."""
    g = synth.rng(8)
    shapes = [([700, 30], [1, 2]), ([9000], [1]), ([130], [130])]
    calls = []
    for lens, rows in shapes:
        c = attn_cases.random_plan(g, lens, rows, 2, 128, "q4_0")
        q = dev(2 * synth.normal_f32(g, (c.T, 8, 128)))
        calls.append((attn_cases.on_gpu(c), q, w4.attn_workspace(attn_cases.on_gpu(c), c.T, 8).numel()))
    ws = torch.zeros(max(n for *_, n in calls), dtype=torch.uint8, device="cuda")
    xs = [torch.randn(t, 20000, device="cuda") for t in (1, 5)]
    lw = torch.zeros(max(w4.logprobs_workspace(x.shape[0], 20000, 7).numel() for x in xs),
                     dtype=torch.uint8, device="cuda")
    run = [lambda kv=kv, q=q: w4.attn_forward(kv, q, 0.09, workspace=ws) for kv, q, _ in calls] + \
          [lambda x=x: w4.token_logprobs(x, None, 7, workspace=lw)[1:] for x in xs]
    want = [[y.clone() for y in f()] for f in run]
    torch.cuda.synchronize()
    graphs, got = [], []
    for f in run:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(f())
    for i in range(4):
        for k in (range(len(run)) if i % 2 else reversed(range(len(run)))):
            for y in got[k]:
                y.fill_(3)
            graphs[k].replay()
            other = run[(k + i) % len(run)]()
            torch.cuda.synchronize()
            for a, b in zip(got[k], want[k]):
                assert torch.equal(a, b), (i, k)
            for a, b in zip(other, want[(k + i) % len(run)]):
                assert torch.equal(a, b), (i, k)
