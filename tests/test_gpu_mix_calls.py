"""Calls of the 8-bit row, convolution and scan entry points that are not about
values: a call's own outputs on another stream, plans whose rows decrease,
offsets past 32 bits (GPU)."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from tests import mix_ref as ref
from tests.test_gpu_own_outputs import check as check_own_outputs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def calls():
    r = lambda *s: torch.randn(*s, device="cuda", generator=torch.Generator("cuda").manual_seed(len(s) + s[0]))
    x, w = r(70, 300), r(200, 300)
    xq, wq = w4.q8_row_quantize(x), w4.q8_row_quantize(w)
    plan = w4.SeqPlan(i32(0, 60, 70), 2, src=i32(-1, -1), dst=i32(-1, -1))
    cx, cw, cs = r(70, 64), r(4, 64), r(2, 3, 64)
    h, b, dt, A, st = r(70, 2, 64), r(70, 1, 64), r(70, 2), -r(2).abs(), r(2, 2, 64, 64)
    return {
        "q8_row_quantize": lambda s: list(w4.q8_row_quantize(x, stream=s)),
        "q8q8_gemm": lambda s: [w4.q8q8_gemm(*xq, *wq, stream=s)],
        "short_conv": lambda s: [w4.short_conv(plan, cx, cw, cs, stream=s)],
        "ssm_scan": lambda s: [w4.ssm_scan(plan, h, dt, A, b, b, st, stream=s)],
    }


@pytest.mark.parametrize("name", ["q8_row_quantize", "q8q8_gemm", "short_conv", "ssm_scan"])
def test_own_outputs_on_another_stream(name):
    check_own_outputs(calls()[name])


def test_plans_whose_rows_decrease_touch_nothing_else():
    """What rows are written is open, but not where: rows and slots that no
    sequence names stay."""
    T = 90
    plan = w4.SeqPlan(i32(10, 60, 20, 200, -5), 6, src=i32(0, 1, -1, 9), dst=i32(2, 3, 1 << 30, -7))
    x, w = torch.randn(T, 64, device="cuda"), torch.randn(4, 64, device="cuda")
    st = torch.full((6, 3, 64), 7.0, device="cuda")
    out = torch.full((T + 64, 64), 7.0, device="cuda")
    w4.short_conv(plan, x, w, st, out=out[:T])
    assert bool((out[:10] == 7).all()) and bool((out[T:] == 7).all()) and bool((st[[0, 1, 4, 5]] == 7).all())
    h, b, dt = torch.randn(T, 2, 64, device="cuda"), torch.randn(T, 1, 64, device="cuda"), torch.rand(T, 2, device="cuda")
    st = torch.full((6, 2, 64, 64), 7.0, device="cuda")
    out = torch.full((T + 64, 2, 64), 7.0, device="cuda")
    w4.ssm_scan(plan, h, dt, -torch.rand(2, device="cuda"), b, b, st, out=out[:T])
    assert bool((out[:10] == 7).all()) and bool((out[T:] == 7).all()) and bool((st[[0, 1, 4, 5]] == 7).all())


# ------------------------------------------------------------------ offsets past 2^31 elements
def test_far_rows_of_the_convolution_and_the_scan():
    """The last rows of a tensor of 2.3e9 elements, against the same rows by
    themselves."""
    T, wide, near = 70000, 33024, 200
    big = torch.empty(T, wide, device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    ends = i32(0, T - near, T)
    tail = torch.randn(near, 512, device="cuda", generator=g)
    big[:, :512] = 0.0
    big[T - near:, :512] = tail
    w, cs = torch.randn(4, 64, device="cuda", generator=g), torch.zeros(1, 3, 64, device="cuda")
    out = torch.empty(T, wide, device="cuda")
    none = i32(-1, -1)
    w4.short_conv(w4.SeqPlan(ends, 1, src=none, dst=i32(-1, 0)), big[:, :64], w, cs, out=out[:, 64:128])
    cs2 = torch.zeros_like(cs)
    want = w4.short_conv(w4.SeqPlan(i32(0, near), 1, src=i32(-1)), tail[:, :64], w, None if cs2 is None else cs2)
    assert torch.equal(out[T - near:, 64:128], want)
    assert torch.equal(cs[0], tail[-3:, :64])
    A = -torch.rand(2, device="cuda", generator=g)
    st, st2 = torch.zeros(1, 2, 64, 64, device="cuda"), torch.zeros(1, 2, 64, 64, device="cuda")
    cut = lambda t: dict(x=t[:, :128].unflatten(1, (2, 64)), dt=t[:, 256:258], B=t[:, 128:192].unflatten(1, (1, 64)),
                         C=t[:, 192:256].unflatten(1, (1, 64)), z=t[:, 384:512].unflatten(1, (2, 64)))
    a = cut(big)
    w4.ssm_scan(w4.SeqPlan(ends, 1, src=none, dst=i32(-1, 0)), a["x"], a["dt"], A, a["B"], a["C"], st, z=a["z"],
                out=out[:, 128:256].unflatten(1, (2, 64)))
    a = cut(tail)
    want = w4.ssm_scan(w4.SeqPlan(i32(0, near), 1, src=i32(-1), dst=i32(0)), a["x"], a["dt"], A, a["B"], a["C"], st2,
                       z=a["z"])
    assert torch.equal(out[T - near:, 128:256], want.flatten(1)) and torch.equal(st, st2)


def test_far_states():
    """Slots past 2^31 elements of the pools."""
    slots = 66000
    st = torch.empty(slots, 4, 64, 128, device="cuda")               # 2.16e9
    st[slots - 1] = 0.0
    h, b = torch.randn(3, 4, 128, device="cuda"), torch.randn(3, 1, 64, device="cuda")
    dt, A = torch.rand(3, 4, device="cuda"), -torch.rand(4, device="cuda")
    small = torch.zeros(1, 4, 64, 128, device="cuda")
    for n in (3, 1):
        y = w4.ssm_scan(w4.SeqPlan(i32(0, n), slots, src=i32(slots - 1)), h[:n], dt[:n], A, b[:n], b[:n], st)
        want = w4.ssm_scan(w4.SeqPlan(i32(0, n), 1), h[:n], dt[:n], A, b[:n], b[:n], small)
        assert torch.equal(y, want) and torch.equal(st[-1:], small)


@pytest.mark.parametrize("M", [1, 70])
def test_far_channels_and_rows_of_the_product(M):
    N, K = 33000, 70000                                              # 2.3e9 codes
    w = torch.randint(-127, 128, (N, 70016), dtype=torch.int8, device="cuda")
    g = np.random.default_rng(M)
    xq = np.zeros((M, 70016), np.int8)
    xq[:, :K] = g.integers(-127, 128, (M, K))
    xd, wd = g.random(M).astype(np.float32), g.random(N).astype(np.float32)
    d = lambda a: torch.from_numpy(a).to("cuda")
    out = torch.empty(M, 33000, device="cuda")
    w4.q8q8_gemm(d(xq), d(xd), w, d(wd), out=out)
    last = [0, 12345, N - 200, N - 2, N - 1]
    want, bound = ref.product(xq, xd, w[last].cpu().numpy(), wd[last])
    assert np.all(np.abs(out[:, last].cpu().numpy() - want) <= bound)


def test_far_rows_of_the_quantizer_and_of_an_output():
    M, K, wide = 70000, 64, 33024
    big = torch.empty(M, wide, device="cuda")
    tail = torch.randn(300, K, device="cuda")
    big[:, 4:4 + K] = 1.0
    big[M - 300:, 4:4 + K] = tail
    q, dd = w4.q8_row_quantize(big[:, 4:4 + K])
    q2, d2 = w4.q8_row_quantize(tail)
    assert torch.equal(q[M - 300:], q2) and torch.equal(dd[M - 300:], d2)
    wq, wd = w4.q8_row_quantize(torch.randn(40, K, device="cuda"))
    w4.q8q8_gemm(q, dd, wq, wd, out=big[:, 100:140])
    assert torch.equal(big[M - 300:, 100:140], w4.q8q8_gemm(q2, d2, wq, wd))
