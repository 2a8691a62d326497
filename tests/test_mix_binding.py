"""What the binding of the 8-bit row, convolution and scan calls refuses, each by
the check of that argument: every refusal names it, where right tensors on the
CPU are refused for their device alone."""
import ctypes

import pytest

import paper_2606_24031_amd as w4
from tests.test_mix_abi import conv_call, scan_call, seqs, ssm

torch = pytest.importorskip("torch")

ON_CPU = "a GPU's are needed"
Z = torch.zeros


def refuses(what, f, *a, **kw):
    with pytest.raises(ValueError, match=what):
        f(*a, **kw)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_quantizer():
    x = Z(4, 200)
    refuses(ON_CPU, w4.q8_row_quantize, x)
    refuses(ON_CPU, w4.q8_row_quantize, Z(4, 240)[:, 8:208], q=Z(4, 256, dtype=torch.int8), d=Z(4))
    for bad in (x.double(), Z(200, 4).t(), x[0], Z(4, 2, 100), Z(4, 400)[:, ::2]):
        refuses("^x: ", w4.q8_row_quantize, bad)
    for q in (Z(4, 200, dtype=torch.int8), Z(3, 256, dtype=torch.int8), Z(4, 256), Z(4, 512, dtype=torch.int8)[:, :256]):
        refuses("^q: ", w4.q8_row_quantize, x, q=q)
    for d in (Z(3), Z(4).double(), Z(8)[::2], Z(4, 1)):
        refuses("^d: ", w4.q8_row_quantize, x, d=d)


def test_product():
    q, d, wq, wd = Z(4, 256, dtype=torch.int8), Z(4), Z(6, 256, dtype=torch.int8), Z(6)
    refuses(ON_CPU, w4.q8q8_gemm, q, d, wq, wd)
    refuses(ON_CPU, w4.q8q8_gemm, q, d, wq, wd, bias=Z(6), out=Z(4, 10)[:, 2:8])
    odd = Z(4, 200, dtype=torch.int8)
    for a in ((q.float(), d), (odd, d), (q[0], d), (Z(4, 512, dtype=torch.int8)[:, :256], d), (q, d[:3]), (q, d.double()),
              (q, d[:, None]), (q, Z(8)[::2])):
        refuses("^xq, xd: ", w4.q8q8_gemm, *a, wq, wd)
        refuses("^wq, wd: ", w4.q8q8_gemm, wq, wd, *a)
    refuses("^xq and wq: ", w4.q8q8_gemm, q, d, Z(6, 384, dtype=torch.int8), wd)
    for bias in (Z(4), Z(6).double(), Z(12)[::2]):
        refuses("^bias: ", w4.q8q8_gemm, q, d, wq, wd, bias=bias)
    for out in (Z(4, 5), Z(5, 6), Z(4, 6).double(), Z(6, 4).t(), Z(24)):
        refuses("^out: ", w4.q8q8_gemm, q, d, wq, wd, out=out)


def test_plan():
    refuses("^cu_rows: ", w4.SeqPlan, Z(3), 4)
    refuses("^cu_rows: ", w4.SeqPlan, i32(), 4)
    refuses("^cu_rows: ", w4.SeqPlan, i32(0, 1, 2, 3)[::2], 4)
    for bad in (i32(0, 1), Z(1), i32(0).long()):
        refuses("^src: ", w4.SeqPlan, i32(0, 4), 4, src=bad)
        refuses("^dst: ", w4.SeqPlan, i32(0, 4), 4, dst=bad)


def test_convolution():
    plan, x, w, st = w4.SeqPlan(i32(0, 2, 4), 3, src=i32(0, 1)), Z(4, 200), Z(4, 200), Z(3, 3, 200)
    refuses(ON_CPU, w4.short_conv, plan, x, w, st)
    refuses(ON_CPU, w4.short_conv, plan, x, w, st, bias=Z(200), out=Z(4, 220)[:, 4:204])
    refuses(ON_CPU, w4.short_conv, w4.SeqPlan(i32(0, 4), 0), x, w, None)
    for bad in (x.double(), Z(200, 4).t(), Z(4, 1, 200)):
        refuses("^x: ", w4.short_conv, plan, bad, w, st)
    for bad in (w[:, :196], Z(4, 196), w.double(), w[0]):
        refuses("^w: ", w4.short_conv, plan, x, bad, st)
    for bad in (None, st[:2], st[:, :2], Z(3, 3, 196), st.double(), Z(3, 3, 400)[..., ::2]):
        refuses("^state: ", w4.short_conv, plan, x, w, bad)
    for bad in (Z(4), Z(200).double(), Z(1, 200)):
        refuses("^bias: ", w4.short_conv, plan, x, w, st, bias=bad)
    for bad in (Z(4, 196), Z(3, 200), Z(4, 200).double(), Z(200, 4).t()):
        refuses("^out: ", w4.short_conv, plan, x, w, st, out=bad)
    refuses("^act ", w4.short_conv, plan, x, w, st, act="relu")


def test_scan():
    plan, h = w4.SeqPlan(i32(0, 2, 4), 3, src=i32(0, 1)), Z(4, 2, 64)
    right = dict(dt=Z(4, 2), A=Z(2), B=Z(4, 1, 64), C=Z(4, 1, 64), state=Z(3, 2, 64, 64))
    ws = Z(1 << 20, dtype=torch.uint8)
    refuses(ON_CPU, w4.ssm_scan, plan, h, **right, workspace=ws)
    refuses(ON_CPU, w4.ssm_scan, plan, h, **right, D=Z(2), z=Z(4, 2, 64), dt_bias=Z(2), out=Z(4, 3, 64)[:, 1:], workspace=ws)
    refuses("^workspace: ", w4.ssm_scan, plan, h, **right, workspace=ws[::2])
    for bad in (h[0], h.double(), Z(4, 64, 2).transpose(1, 2), Z(4, 2, 128)[..., ::2], Z(4, 2, 80)[..., :64]):
        refuses("^x: ", w4.ssm_scan, plan, bad, **right)
    vector = (Z(3), Z(1), Z(2).double(), Z(2, 1), Z(4)[::2])
    for name, bads in dict(
            dt=(Z(4, 3), Z(3, 2), Z(4, 2).double(), Z(2, 4).t(), Z(4, 2, 1)),
            A=vector, D=vector, dt_bias=vector,
            B=(Z(3, 1, 64), Z(4, 64), Z(4, 1, 64).double(), Z(4, 1, 128)[..., ::2], Z(4, 2, 80)[..., :64]),
            C=(Z(3, 1, 64), Z(4, 64), Z(4, 1, 64).double(), Z(4, 1, 128), Z(4, 2, 64)),
            state=(None, Z(2, 2, 64, 64), Z(3, 1, 64, 64), Z(3, 2, 64, 32), Z(3, 2, 32, 64), Z(3, 2, 64, 64).double(),
                   Z(3, 2, 64, 64).transpose(2, 3)),
            z=(Z(4, 1, 64), Z(3, 2, 64), Z(4, 2, 32), Z(4, 2, 64).double(), Z(4, 128)),
            out=(Z(4, 2, 32), Z(3, 2, 64), Z(4, 2, 64).double(), Z(4, 2, 80)[..., :64])).items():
        for bad in bads:
            refuses(f"^{name}: ", w4.ssm_scan, plan, h, **{**right, name: bad}, workspace=ws)


def test_sizes_out_of_range_are_out_of_range_alone():
    """Each range by itself, all else right."""
    wide = dict(x_stride=1 << 23, z_stride=1 << 23, dt_stride=1 << 17, b_stride=1 << 23, c_stride=1 << 23)
    for kw in (dict(NH=1 << 16, P=16, **wide), dict(P=4112, **wide), dict(x_stride=1 << 24), dict(b_stride=1 << 24),
               dict(c_stride=1 << 24), dict(dt_stride=1 << 24), dict(z_stride=1 << 24)):
        assert scan_call(m=ssm(**kw), ys=1 << 23) == w4.ERANGE, kw
    ok = dict(NH=(1 << 16) - 1, P=16, **wide)
    assert scan_call(m=ssm(**ok), ys=1 << 23, T=0) == w4.OK
    # rows times channels of the convolution
    assert conv_call(T=1 << 20, CH=1 << 20, xs=1 << 20, os=1 << 20) == w4.ERANGE
    assert conv_call(T=(1 << 20) - 1, CH=1 << 20, xs=1 << 20, os=1 << 20, q=seqs(B=0)) == w4.OK
    assert w4.lib().ssm_workspace_size(ctypes.byref(seqs()), ctypes.byref(ssm(**ok)), 4) > 0
