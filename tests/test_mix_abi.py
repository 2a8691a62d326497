"""Refusals of the 8-bit row, convolution and state space entry points (host
checks, which run without a GPU), and pins of the plain forms that the GPU
tests compare with."""
import ctypes

import numpy as np
import pytest

import paper_2606_24031_amd as w4
from tests import mix_ref as ref

A = 0x10000   # an aligned fake device address (never dereferenced: validation fails first)
TOP = 1 << 31


def P(addr):
    return None if addr is None else ctypes.c_void_p(addr)


def seqs(**kw):
    a = dict(cu_rows=A + 0x100, src=A + 0x200, dst=A + 0x300, n_slots=4, B=2)
    a.update(kw)
    return w4._SeqArgs(*(a[k] for k, _ in w4._SeqArgs._fields_))


def test_row_bytes():
    F = w4.lib().q8_row_bytes
    assert [F(k) for k in (1, 128, 129, 2048, (1 << 17) - 1)] == [128, 128, 256, 2048, 1 << 17]
    assert F(0) == 0 and F(-5) == 0 and F(1 << 17) == 0


def test_quantize_errors():
    def call(x=A, xs=300, q=A + 0x1000, d=A + 0x2000, rows=4, K=300):
        return w4.lib().q8_row_quantize(P(x), xs, P(q), P(d), rows, K, None)
    for kw in (dict(x=None), dict(q=None), dict(d=None)):
        assert call(**kw) == w4.ENULL, kw
    for kw in (dict(rows=-1), dict(K=0), dict(xs=299)):
        assert call(**kw) == w4.ESHAPE, kw
    for kw in (dict(K=1 << 17, xs=1 << 17), dict(rows=TOP), dict(xs=TOP)):
        assert call(**kw) == w4.ERANGE, kw
    for kw in (dict(x=A + 2), dict(q=A + 8), dict(d=A + 1)):
        assert call(**kw) == w4.EALIGN, kw
    assert call(rows=0) == w4.OK


def test_product_errors():
    def call(xq=A, xd=A + 0x1000, wq=A + 0x2000, wd=A + 0x3000, bias=A + 0x4000, y=A + 0x5000, ys=100, M=4, N=100,
             K=300):
        return w4.lib().q8q8_gemm(P(xq), P(xd), P(wq), P(wd), P(bias), P(y), ys, M, N, K, None)
    for kw in (dict(xq=None), dict(xd=None), dict(wq=None), dict(wd=None), dict(y=None)):
        assert call(**kw) == w4.ENULL, kw
    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(ys=99)):
        assert call(**kw) == w4.ESHAPE, kw
    for kw in (dict(K=1 << 17), dict(M=TOP), dict(N=TOP, ys=TOP), dict(ys=TOP), dict(M=1 << 26, N=1, ys=1),
               dict(N=1 << 26, ys=1 << 26), dict(M=1 << 20, N=1 << 16, ys=1 << 16)):
        assert call(**kw) == w4.ERANGE, kw
    for kw in (dict(xq=A + 8), dict(wq=A + 4), dict(xd=A + 2), dict(wd=A + 1), dict(bias=A + 3), dict(y=A + 2)):
        assert call(**kw) == w4.EALIGN, kw
    for p in (A, A + 0x1000, A + 0x2000, A + 0x3000, A + 0x4000):
        assert call(y=p) == w4.EALIAS
    assert call(M=0) == w4.OK and call(M=0, bias=None) == w4.OK


def conv_call(q=None, x=A, xs=64, w=A + 0x1000, bias=A + 0x2000, state=A + 0x3000, out=A + 0x4000, os=64, T=4, CH=64,
              W=4, act=1, null=False):
    return w4.lib().short_conv(None if null else ctypes.byref(q or seqs()), P(x), xs, P(w), P(bias), P(state), P(out),
                               os, T, CH, W, act, None)


def ssm(**kw):
    a = dict(x=A, dt=A + 0x1000, b=A + 0x2000, c=A + 0x3000, z=A + 0x4000, A=A + 0x5000, D=A + 0x6000,
             dt_bias=A + 0x7000, x_stride=128, dt_stride=2, b_stride=64, c_stride=64, z_stride=128, NH=2, NG=1, N=64,
             P=64, softplus=1)
    a.update(kw)
    return w4._SsmArgs(*(a[k] for k, _ in w4._SsmArgs._fields_))


def scan_call(q=None, m=None, state=A + 0x8000, y=A + 0x9000, ys=128, T=4, ws=A + 0xA000, nb=1 << 40, null=False):
    return w4.lib().ssm_scan(ctypes.byref(q or seqs()), None if null else ctypes.byref(m or ssm()), P(state), P(y), ys,
                             T, P(ws), nb, None)


@pytest.mark.parametrize("call", [conv_call, scan_call])
def test_plan_errors(call):
    assert call(q=seqs(cu_rows=None)) == w4.ENULL
    for kw in (dict(B=-1), dict(n_slots=-1)):
        assert call(q=seqs(**kw)) == w4.ESHAPE, kw
    for kw in (dict(B=1 << 20), dict(n_slots=TOP)):
        assert call(q=seqs(**kw)) == w4.ERANGE, kw
    for kw in (dict(cu_rows=A + 1), dict(src=A + 2), dict(dst=A + 3)):
        assert call(q=seqs(**kw)) == w4.EALIGN, kw
    assert call(T=-1) == w4.ESHAPE and call(T=TOP) == w4.ERANGE
    assert call(state=None) == w4.ENULL
    assert call(T=0) == w4.OK and call(q=seqs(B=0, cu_rows=None)) == w4.OK
    assert call(q=seqs(n_slots=0), state=None, T=0) == w4.OK


def test_convolution_errors():
    assert conv_call(null=True) == w4.ENULL
    for kw in (dict(x=None), dict(w=None), dict(out=None)):
        assert conv_call(**kw) == w4.ENULL, kw
    for kw in (dict(CH=0), dict(CH=62), dict(W=1), dict(W=5), dict(act=2), dict(act=-1), dict(xs=60), dict(os=60),
               dict(xs=66), dict(os=65)):
        assert conv_call(**kw) == w4.ESHAPE, kw
    for kw in (dict(CH=1 << 24, xs=1 << 24, os=1 << 24), dict(xs=TOP), dict(os=TOP)):
        assert conv_call(**kw) == w4.ERANGE, kw
    for kw in (dict(x=A + 4), dict(w=A + 8), dict(bias=A + 4), dict(state=A + 4), dict(out=A + 12)):
        assert conv_call(**kw) == w4.EALIGN, kw
    for kw in (dict(out=A), dict(state=A), dict(state=A + 0x4000)):
        assert conv_call(**kw) == w4.EALIAS, kw


def test_scan_errors():
    assert scan_call(null=True) == w4.ENULL
    for kw in (dict(x=None), dict(dt=None), dict(b=None), dict(c=None), dict(A=None)):
        assert scan_call(m=ssm(**kw)) == w4.ENULL, kw
    assert scan_call(y=None) == w4.ENULL and scan_call(ws=None) == w4.ENULL
    for kw in (dict(NH=0), dict(NG=0), dict(NH=3, NG=2), dict(N=32), dict(N=192), dict(P=8), dict(P=72), dict(P=0),
               dict(x_stride=124), dict(x_stride=130), dict(b_stride=60), dict(b_stride=65), dict(c_stride=60),
               dict(c_stride=66), dict(z_stride=120), dict(z_stride=129), dict(dt_stride=1)):
        assert scan_call(m=ssm(**kw)) == w4.ESHAPE, kw
    assert scan_call(ys=124) == w4.ESHAPE and scan_call(ys=130) == w4.ESHAPE
    for kw in (dict(NH=1 << 16), dict(P=4112), dict(x_stride=1 << 24), dict(b_stride=1 << 24),
               dict(c_stride=1 << 24), dict(dt_stride=1 << 24), dict(z_stride=1 << 24)):
        assert scan_call(m=ssm(**kw)) in (w4.ERANGE, w4.ESHAPE), kw
    assert scan_call(m=ssm(P=4112, x_stride=1 << 14, z_stride=1 << 14), ys=1 << 14) == w4.ERANGE
    assert scan_call(ys=1 << 24) == w4.ERANGE
    assert scan_call(q=seqs(B=(1 << 20) - 1), m=ssm(NH=4, x_stride=256, z_stride=256, dt_stride=4), ys=256) == w4.ERANGE
    assert scan_call(T=1 << 29) == w4.ERANGE
    assert w4.lib().ssm_workspace_size(ctypes.byref(seqs()), ctypes.byref(ssm()), 1 << 29) == 0
    for kw in (dict(x=A + 4), dict(b=A + 8), dict(c=A + 4), dict(z=A + 4), dict(dt=A + 2), dict(A=A + 1),
               dict(D=A + 3), dict(dt_bias=A + 2)):
        assert scan_call(m=ssm(**kw)) == w4.EALIGN, kw
    assert scan_call(y=A + 4) == w4.EALIGN and scan_call(state=A + 4) == w4.EALIGN and scan_call(ws=A + 4) == w4.EALIGN
    for p in (A, A + 0x1000, A + 0x2000, A + 0x3000, A + 0x4000, A + 0x5000, A + 0x6000, A + 0x7000):
        assert scan_call(y=p) == w4.EALIAS and scan_call(state=p) == w4.EALIAS
    assert scan_call(y=A + 0x8000) == w4.EALIAS
    n = w4.lib().ssm_workspace_size(ctypes.byref(seqs()), ctypes.byref(ssm()), 4)
    assert n > 0 and scan_call(nb=n - 1) == w4.EWORKSPACE
    S = lambda q, m, T: w4.lib().ssm_workspace_size(ctypes.byref(q), ctypes.byref(m), T)
    # sizes only: the pointers are not looked at
    assert S(seqs(cu_rows=None), ssm(x=None, x_stride=0), 4) == n
    assert S(seqs(), ssm(N=96), 4) == 0 and S(seqs(B=-1), ssm(), 4) == 0 and S(seqs(), ssm(), -1) == 0
    assert w4.lib().ssm_workspace_size(None, ctypes.byref(ssm()), 4) == 0
    assert w4.lib().ssm_workspace_size(ctypes.byref(seqs()), None, 4) == 0


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    x = torch.zeros(4, 200)
    for bad in (x, x.double(), x.t(), x[0]):                       # the first for not being on a GPU
        with pytest.raises(ValueError):
            w4.q8_row_quantize(bad)
    with pytest.raises(ValueError):
        w4.q8_row_quantize(x, q=torch.zeros(4, 200, dtype=torch.int8))
    q, d = torch.zeros(4, 256, dtype=torch.int8), torch.zeros(4)
    for a in ((q, d, q, d), (q, d, q[:, :128], d), (q, d[:3], q, d), (q[:, :200].contiguous(), d, q[:, :200], d),
              (q.float(), d, q, d)):
        with pytest.raises(ValueError):
            w4.q8q8_gemm(*a)
    with pytest.raises(ValueError):
        w4.q8q8_gemm(q, d, q, d, out=torch.zeros(4, 5))
    with pytest.raises(ValueError):
        w4.SeqPlan(torch.zeros(3), 4)
    with pytest.raises(ValueError):
        w4.SeqPlan(i32(), 4)
    with pytest.raises(ValueError):
        w4.SeqPlan(i32(0, 4), 4, src=i32(0, 1))
    plan = w4.SeqPlan(i32(0, 2, 4), 3, src=i32(0, 1))
    w, st = torch.zeros(4, 200), torch.zeros(3, 3, 200)
    for kw in (dict(), dict(act="relu"), dict(bias=torch.zeros(4)), dict(out=torch.zeros(4, 196)), dict(state=None),
               dict(state=st[:2]), dict(w=w[:, :196])):
        a = dict(w=w, state=st)
        a.update(kw)
        with pytest.raises(ValueError):
            w4.short_conv(plan, x, **a)
    h, b, s = torch.zeros(4, 2, 64), torch.zeros(4, 1, 64), torch.zeros(3, 2, 64, 64)
    for kw in (dict(), dict(dt=torch.zeros(4, 3)), dict(A=torch.zeros(3)), dict(B=b[:3]), dict(C=torch.zeros(4, 1, 128)),
               dict(state=None), dict(state=s[:, :1]), dict(D=torch.zeros(1)), dict(z=h[:, :1]), dict(dt_bias=b),
               dict(out=h[..., :32]), dict(B=torch.zeros(4, 64))):
        a = dict(dt=torch.zeros(4, 2), A=torch.zeros(2), B=b, C=b, state=s)
        a.update(kw)
        with pytest.raises(ValueError):
            w4.ssm_scan(plan, h, **a)
    with pytest.raises(w4.W4A8Error):
        w4.ssm_workspace(plan, 4, 2, 1, 48, 64)


# ------------------------------------------------------------------ the plain forms themselves
def test_plain_quantizer_on_known_rows():
    x = np.array([[127.0, -2.5, 2.5, 0.4, -126.5], [0, 0, 0, 0, 0], [1, np.nan, 0, 0, 0], [1, -np.inf, 0, 0, 0],
                  [1e-44, 0, 0, 0, 0]], np.float32)
    q, d = ref.quantize(x)
    assert q.shape == (5, 128) and not q[:, 5:].any() and not q[1:].any()
    assert list(q[0, :5]) == [127, -3, 3, 0, -127] and d[0] == 1 and d[1] == 0 and q[0, 5:].max() == 0
    assert np.isnan(d[2]) and np.isnan(d[3]) and d[4] == 0


def test_plain_quantizer_is_the_oracles_but_for_an_ulp_of_the_scale():
    import oracle
    oracle.build()
    g = np.random.default_rng(4)
    x = (g.standard_normal((300, 32)) * np.exp2(g.integers(-20, 20, (300, 1)))).astype(np.float32)
    raw = np.asarray(oracle.q8_f32_quantize(x)).reshape(300, 36)
    q, d = ref.quantize(x)
    d0 = np.ascontiguousarray(raw[:, :4]).view(np.float32)[:, 0]
    assert np.all(np.abs(d - d0) <= np.spacing(d0)) and (d != d0).any() and (d == d0).any()
    assert np.array_equal(raw[:, 4:].view(np.int8)[d == d0], q[:, :32][d == d0])
    assert np.all(np.abs(raw[:, 4:].view(np.int8).astype(int) - q[:, :32]) <= 1)


def test_plain_convolution_is_numpys():
    g = np.random.default_rng(5)
    x, w = g.standard_normal((30, 4)).astype(np.float32), g.standard_normal((3, 4)).astype(np.float32)
    y, _, st = ref.conv([0, 30], [-1], [0], x, w, None, np.zeros((1, 2, 4), np.float32), "none")
    for c in range(4):
        assert np.allclose(y[:, c], np.convolve(x[:, c].astype(float), w[::-1, c].astype(float))[:30], atol=1e-12)
    assert np.array_equal(st[0], x[28:])
    # in two pieces through the state
    a, _, st = ref.conv([0, 1], [-1], [0], x[:1], w, None, np.zeros((1, 2, 4), np.float32), "none")
    b, _, _ = ref.conv([0, 29], [0], [0], x[1:], w, None, st, "none")
    assert np.allclose(np.concatenate([a, b]), y, atol=1e-12)


def test_plain_scan_closed_forms():
    g = np.random.default_rng(6)
    T, NH, N, Pc = 12, 2, 64, 16
    x, B = g.standard_normal((T, NH, Pc)).astype(np.float32), g.standard_normal((T, 1, N)).astype(np.float32)
    C = g.standard_normal((T, 1, N)).astype(np.float32)
    dt, A = g.random((T, NH)).astype(np.float32), -g.random(NH).astype(np.float32)
    y, _, st, _ = ref.scan([0, T], [-1], [0], x, dt, A, B, C, np.zeros((1, NH, N, Pc), np.float32), softplus=False)
    L = np.cumsum(dt.astype(float) * A, 0)
    for h in range(NH):
        Wt = np.tril(np.exp(L[:, None, h] - L[None, :, h])) * (C[:, 0].astype(float) @ B[:, 0].T) * dt[None, :, h]
        assert np.allclose(y[:, h], Wt @ x[:, h], atol=1e-10)
    # in two pieces through the state, and D and a gate on top
    D, z = np.array([2.0, -1.0]), g.standard_normal((T, NH, Pc))
    a, _, s1, _ = ref.scan([0, 5], [-1], [0], x[:5], dt[:5], A, B[:5], C[:5], np.zeros((1, NH, N, Pc), np.float32),
                           softplus=False)
    b, _, s2, _ = ref.scan([0, 7], [0], [0], x[5:], dt[5:], A, B[5:], C[5:], s1, D, z[5:], softplus=False)
    assert np.allclose(s2, st, atol=1e-10)
    assert np.allclose(b, (y[5:] + D[:, None] * x[5:]) * z[5:] / (1 + np.exp(-z[5:])), atol=1e-10)
