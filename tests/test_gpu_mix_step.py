"""A state space layer run as a served model runs it: the projection in 8 bits,
the convolution, the scan, the norm, the projection back; a prompt, then tokens;
eagerly, replayed from graphs, on streams of their own; and the convolution in
front of the gated delta rule (GPU).  Each operator is checked on the inputs that
it got, within its own bounds (tests/mix_ref.py)."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from oracle.gdn import gdn_recurrent
from tests import mix_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

H, NH, P, N, NG, W = 256, 4, 64, 64, 2, 4
XB = NH * P + 2 * NG * N            # convolved channels
ROW = NH * P + XB + NH              # the projection's: z, the convolved ones, dt


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def i32(a):
    return dev(np.asarray(a, np.int32))


class Layer:
    def __init__(self, seed):
        g = np.random.default_rng(seed)
        f = lambda *s: dev(g.standard_normal(s).astype(np.float32))
        self.w_in = w4.q8_row_quantize(f(ROW, H) / H ** 0.5)
        self.w_out = w4.q8_row_quantize(f(H, NH * P) / (NH * P) ** 0.5)
        self.conv, self.bias, self.gamma = f(W, XB) / 2, 0.1 * f(XB), 1 + 0.1 * f(NH * P)
        self.A, self.D, self.dt_bias = -1 - 15 * f(NH).abs(), f(NH), f(NH) - 4


class Session:
    """States of `slots` slots, and a layer's run over them.  Buffers of a step
    are made once, so that a graph can hold it."""

    def __init__(self, layer, slots, seed=0):
        self.m, self.slots = layer, slots
        self.cs = torch.full((slots, W - 1, XB), float("nan"), device="cuda")
        self.ss = torch.full((slots, NH, N, P), float("nan"), device="cuda")

    def step(self, hidden, cu, src, dst, stream=None, ws=None, keep=None):
        m = self.m
        plan = w4.SeqPlan(cu, self.slots, src=src, dst=dst)
        T = hidden.shape[0]
        k = dict(stream=stream)
        xq, xd = w4.q8_row_quantize(hidden, **k)
        row = w4.q8q8_gemm(xq, xd, *m.w_in, **k)
        z, xbc, dt = row[:, :NH * P], row[:, NH * P:NH * P + XB], row[:, NH * P + XB:]
        if keep is not None:
            keep.update(cs0=self.cs.clone(), ss0=self.ss.clone())
        c = w4.short_conv(plan, xbc, m.conv, self.cs, bias=m.bias, **k)
        x, b, cc = c[:, :NH * P], c[:, NH * P:NH * P + NG * N], c[:, NH * P + NG * N:]
        y = w4.ssm_scan(plan, x.unflatten(1, (NH, P)), dt, m.A, b.unflatten(1, (NG, N)), cc.unflatten(1, (NG, N)),
                        self.ss, D=m.D, z=z.unflatten(1, (NH, P)), dt_bias=m.dt_bias, workspace=ws, **k)
        _, yn = w4.rmsnorm_residual(y.flatten(1), None, m.gamma, **k)
        yq, yd = w4.q8_row_quantize(yn, **k)
        out = w4.q8q8_gemm(yq, yd, *m.w_out, **k)
        if keep is not None:
            keep.update(xq=xq, xd=xd, row=row, conv=c, y=y, yn=yn, yq=yq, yd=yd, out=out)
        return out

    def check(self, hidden, cu, src, dst, k):
        m, n = self.m, lambda t: t.cpu().numpy()
        q, d = ref.quantize(n(hidden))
        assert np.array_equal(n(k["xq"]), q) and np.array_equal(n(k["xd"]), d)
        want, bound = ref.product(q, d, *map(n, m.w_in))
        assert np.all(np.abs(n(k["row"]) - want) <= bound)
        row, c = n(k["row"]), n(k["conv"])
        want, bound, new = ref.conv(n(cu), n(src), n(dst), row[:, NH * P:NH * P + XB], n(m.conv), n(m.bias), n(k["cs0"]),
                                    "silu")
        assert np.all(np.abs(c - want) <= bound)
        assert np.array_equal(n(self.cs), new, equal_nan=True)
        T = len(row)
        with np.errstate(invalid="ignore"):
            want, by, new, bs = ref.scan(n(cu), n(src), n(dst), c[:, :NH * P].reshape(T, NH, P), row[:, NH * P + XB:],
                                         n(m.A), c[:, NH * P:NH * P + NG * N].reshape(T, NG, N),
                                         c[:, NH * P + NG * N:].reshape(T, NG, N), n(k["ss0"]), n(m.D),
                                         row[:, :NH * P].reshape(T, NH, P), n(m.dt_bias))
        assert np.all(np.abs(n(k["y"]) - want) <= by)
        used = ~np.isnan(new)
        assert np.all((np.abs(n(self.ss) - new) <= bs)[used]) and np.isnan(n(self.ss)[~used]).all()
        q, d = ref.quantize(n(k["yn"]))
        assert np.array_equal(n(k["yq"]), q) and np.array_equal(n(k["yd"]), d)
        want, bound = ref.product(q, d, *map(n, m.w_out))
        assert np.all(np.abs(n(k["out"]) - want) <= bound)


def rows(g, T):
    return dev(g.standard_normal((T, H)).astype(np.float32))


def test_prompts_then_tokens_then_both():
    g = np.random.default_rng(1)
    s = Session(Layer(1), 5)
    for lens, src, dst in (([150, 7], [-1, -1], [3, 0]),           # prompts
                           ([1, 1], [3, 0], [3, 0]),               # a token each
                           ([1, 70, 4], [0, -1, 3], [0, 1, 4]),    # a token, a new prompt, drafts kept elsewhere
                           ([1, 2, 1], [3, 4, 1], [3, 4, 1]),      # from before the drafts and from behind them
                           ([1] * 4, [0, 1, 3, 4], [0, -1, 3, 2])):
        h = rows(g, sum(lens))
        cu, k = i32(np.concatenate([[0], np.cumsum(lens)])), {}
        s.step(h, cu, i32(src), i32(dst), keep=k)
        s.check(h, cu, i32(src), i32(dst), k)


def test_drafts_that_are_not_kept_leave_the_states():
    g = np.random.default_rng(2)
    s = Session(Layer(2), 2)
    s.step(rows(g, 30), i32([0, 30]), i32([-1]), i32([0]))
    before = s.cs.clone(), s.ss.clone()
    h = rows(g, 5)
    out = s.step(h, i32([0, 5]), i32([0]), i32([-1]))
    assert torch.equal(s.cs[0], before[0][0]) and torch.equal(s.ss[0], before[1][0])
    # taken again in two pieces, row by row as before: equal bits
    a = s.step(h[:3], i32([0, 3]), i32([0]), i32([0]))
    b = s.step(h[3:], i32([0, 2]), i32([0]), i32([0]))
    assert torch.equal(torch.cat([a, b]), out)


@pytest.mark.parametrize("lens", [[1, 1, 1], [2, 1, 70]])
def test_replayed_from_a_graph(lens):
    """A captured step replayed as its inputs, sequences and states change, with
    eager work and synchronizations between, against the eager step."""
    g = np.random.default_rng(3)
    layer, B = Layer(3), len(lens)
    a, b = Session(layer, 2 * B), Session(layer, 2 * B)
    T = sum(lens)
    first = rows(g, 10 * B)
    cu0 = i32(10 * np.arange(B + 1))
    for s in (a, b):
        s.step(first, cu0, i32([-1] * B), i32(range(B)))
    h = torch.zeros(T, H, device="cuda")
    cu, src, dst = i32(np.concatenate([[0], np.cumsum(lens)])), i32(range(B)), i32(range(B))
    ws = w4.ssm_workspace(w4.SeqPlan(cu, 2 * B), T, NH, NG, N, P)
    saved = a.cs.clone(), a.ss.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step(h, cu, src, dst, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = a.step(h, cu, src, dst, ws=ws)
    a.cs.copy_(saved[0]), a.ss.copy_(saved[1])
    for i in range(4):
        new = rows(g, T)
        order = g.permutation(lens)
        h.copy_(new)
        cu.copy_(i32(np.concatenate([[0], np.cumsum(order)])))
        src.copy_(i32(g.permutation(B)))
        dst.copy_(src)
        graph.replay()
        got = out.clone()
        want = b.step(new, cu, src, dst)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a.cs[:B], b.cs[:B]) and torch.equal(a.ss[:B], b.ss[:B])
        torch.ones(1000, device="cuda").sum().item()


def test_two_graphs_share_a_workspace_one_after_the_other():
    g = np.random.default_rng(4)
    layer = Layer(4)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    runs = []
    for T in (130, 75):
        s = Session(layer, 1)
        h, cu = rows(g, T), i32([0, T])
        want = s.step(h, cu, i32([-1]), i32([0]))
        graph = torch.cuda.CUDAGraph()
        none, zero = i32([-1]), i32([0])
        with torch.cuda.graph(graph):
            out = s.step(h, cu, none, zero, ws=ws)
        runs.append((graph, out, want, (s, h, cu, none, zero)))
    for _ in range(3):
        for graph, out, want, _ in runs:
            out.zero_()
            graph.replay()
            assert torch.equal(out, want)


def test_two_streams_at_once():
    """Two sessions at once, each on a stream of its own with its own outputs
    and workspace, against one after the other."""
    g = np.random.default_rng(5)
    layer = Layer(5)
    a, b = [Session(layer, 1) for _ in range(2)], [Session(layer, 1) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    none, zero = i32([-1]), i32([0])
    steps = [(n, rows(g, n), rows(g, n), i32([0, n])) for n in (300, 1, 5, 64, 1)]
    want = [[s.step(h, cu, none if j == 0 else zero, zero) for s, h in zip(b, (h0, h1))]
            for j, (n, h0, h1, cu) in enumerate(steps)]
    torch.cuda.synchronize()
    got = []
    for j, (n, h0, h1, cu) in enumerate(steps):
        got.append([s.step(h, cu, none if j == 0 else zero, zero, stream=st)
                    for s, h, st in zip(a, (h0, h1), streams)])
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert all(torch.equal(u, v) for u, v in zip(x, y))
    assert all(torch.equal(s.ss, t.ss) and torch.equal(s.cs, t.cs) for s, t in zip(a, b))


def test_convolution_in_front_of_the_gated_delta_rule():
    """q, k and v of a linear-attention layer convolved together, then the
    library's other recurrence: a prompt in one piece, and cut in two with both
    states handed over."""
    g = np.random.default_rng(6)
    T, heads, D = 90, 2, 64
    CH = 3 * heads * D
    f = lambda *s: dev(g.standard_normal(s).astype(np.float32))
    x, w, gate, beta = f(T, CH), f(W, CH) / 2, -f(T, heads).abs() / 10, torch.sigmoid(f(T, heads))
    norm = lambda t: (t / t.norm(dim=-1, keepdim=True)).contiguous()

    def run(pieces):
        cs, st, out, at = torch.zeros(1, W - 1, CH, device="cuda"), None, [], 0
        for n in pieces:
            r = slice(at, at + n)
            y = w4.short_conv(w4.SeqPlan(i32([0, n]), 1, src=i32([-1 if at == 0 else 0]), dst=i32([0])), x[r], w, cs)
            q, k, v = (t.unflatten(1, (heads, D)) for t in y.split(heads * D, 1))
            a = norm(q), norm(k), v.contiguous(), gate[r].contiguous(), beta[r].contiguous()
            o, st = w4.gdn_scan(*a, s0=st)
            out.append((o, *a))
            at += n
        return [torch.cat(t) for t in zip(*out)], st, cs

    one, two = run([T]), run([41, 49])
    assert torch.equal(one[2], two[2]) and all(torch.equal(a, b) for a, b in zip(one[0][1:], two[0][1:]))
    # each within the recurrence's own bound: 2e-6 of a state column's largest norm (queries of norm 1)
    o, st, smax = gdn_recurrent(*(t.cpu().numpy() for t in one[0][1:]), None)
    for got in (one, two):
        assert np.all(np.abs(got[0][0].cpu().numpy() - o) <= 2.001e-6 * smax[None] + 1e-30)
        assert np.all(np.abs(got[1].cpu().numpy() - st) <= 2.001e-6 * smax[:, None] + 1e-30)
    want, bound, _ = ref.conv([0, T], [-1], [0], x.cpu().numpy(), w.cpu().numpy(), None,
                              np.zeros((1, W - 1, CH), np.float32), "silu")
    y = w4.short_conv(w4.SeqPlan(i32([0, T]), 0), x, w, None).cpu().numpy()
    assert np.all(np.abs(y - want) <= bound)
