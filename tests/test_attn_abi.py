"""Refusals of the rotary, cache, attention and log-probability entry points
(host checks, which run without a GPU), and pins of the plain forms the GPU
tests compare with."""
import ctypes
import math

import numpy as np
import pytest

import paper_2606_24031_amd as w4
from tests import attn_ref as ref

A = 0x10000   # an aligned fake device address (never dereferenced: validation fails first)
NAN, INF = float("nan"), float("inf")


def P(addr):
    return ctypes.c_void_p(addr)


def rope(**kw):
    a = dict(inv_freq=A, pos=A + 0x1000, n_rot=64, layout=0, mscale=1.0)
    a.update(kw)
    return w4._RopeArgs(a["inv_freq"], a["pos"], a["n_rot"], a["layout"], a["mscale"])


def plan(**kw):
    a = dict(k_pages=A, v_pages=A + 0x1000, page_table=A + 0x2000, kv_len=A + 0x3000,
             cu_rows=A + 0x4000, n_pages=8, max_pages=4, B=2, NKV=2, D=128, format=0)
    a.update(kw)
    return w4._KvArgs(*(a[k] for k, _ in w4._KvArgs._fields_))


def test_rope_frequencies_errors():
    F = w4.lib().rope_frequencies
    ok = lambda p=P(A), n=64, base=1e4, kind=0, f=8.0, o=4096.0, fast=32.0, slow=1.0: \
        F(p, n, base, kind, f, o, fast, slow, None)
    assert ok(p=None) == w4.ENULL
    assert ok(p=P(A + 4)) == w4.EALIGN
    for kw in (dict(n=63), dict(n=0), dict(base=1.0), dict(base=INF), dict(base=NAN), dict(kind=3),
               dict(kind=-1), dict(kind=1, f=0.0), dict(kind=1, f=NAN), dict(kind=2, o=0.0),
               dict(kind=2, slow=0.0), dict(kind=2, fast=0.5), dict(kind=2, o=INF),
               dict(kind=2, fast=NAN)):
        assert ok(**kw) == w4.ESHAPE, kw
    assert ok(n=1026) == w4.ERANGE


def test_rope_rotate_errors():
    F = w4.lib().rope_rotate
    def call(r=None, x=P(A), xs=512, o=P(A + 0x8000), os=512, T=4, NH=4, D=128, null=False):
        return F(None if null else ctypes.byref(r or rope()), x, xs, o, os, T, NH, D, None)
    assert call(null=True) == w4.ENULL and call(x=None) == w4.ENULL and call(o=None) == w4.ENULL
    assert call(rope(pos=None)) == w4.ENULL and call(rope(inv_freq=None)) == w4.ENULL
    for r in (rope(n_rot=0), rope(n_rot=63), rope(n_rot=130), rope(layout=2), rope(mscale=INF)):
        assert call(r) == w4.ESHAPE
    for kw in (dict(D=2), dict(D=126), dict(NH=0), dict(T=-1), dict(xs=511), dict(os=508),
               dict(xs=514)):
        assert call(**kw) == w4.ESHAPE, kw
    assert call(D=1028, xs=1 << 20, os=1 << 20) == w4.ERANGE
    assert call(T=1 << 31) == w4.ERANGE and call(xs=1 << 31) == w4.ERANGE
    assert call(x=P(A + 4)) == w4.EALIGN and call(rope(pos=A + 2)) == w4.EALIGN
    assert call(o=P(A), os=516) == w4.EALIAS
    assert call(T=0) == w4.OK


def test_plan_errors():
    L = w4.lib()
    assert L.kv_q4_tile_bytes(128, 0) == 4 * 1024 + 4 * 64 * 2
    assert L.kv_q4_tile_bytes(256, 1) == 8 * 1024 + 8 * 64 * 4
    assert L.kv_q4_tile_bytes(96, 0) == 0 and L.kv_q4_tile_bytes(128, 2) == 0
    read = lambda kv, T=4, k=P(A + 0x8000), v=P(A + 0x9000): \
        L.kv_q4_read(None if kv is None else ctypes.byref(kv), k, v, T, None)
    app = lambda kv: L.kv_q4_append(ctypes.byref(kv), None, P(A), 256, P(A), 256, None, 0, None, 0,
                                    4, None)
    att = lambda kv: L.attn_q4_forward(ctypes.byref(kv), P(A), 512, P(A + 0x8000), None, 4, 4, 0.1,
                                       0, P(A + 0x10000), 1 << 40, None)
    assert read(None) == w4.ENULL
    for f in (read, app, att):
        for kw in (dict(k_pages=None), dict(v_pages=None), dict(page_table=None), dict(kv_len=None),
                   dict(cu_rows=None)):
            assert f(plan(**kw)) == w4.ENULL, kw
        for kw in (dict(D=96), dict(D=512), dict(NKV=0), dict(B=-1), dict(n_pages=-1),
                   dict(max_pages=-1), dict(format=2)):
            assert f(plan(**kw)) == w4.ESHAPE, kw
        for kw in (dict(B=1 << 20), dict(n_pages=1 << 31), dict(max_pages=1 << 24)):
            assert f(plan(**kw)) == w4.ERANGE, kw
        for kw in (dict(k_pages=A + 8), dict(v_pages=A + 4), dict(kv_len=A + 2), dict(cu_rows=A + 1)):
            assert f(plan(**kw)) == w4.EALIGN, kw
    assert read(plan(), T=-1) == w4.ESHAPE and read(plan(), T=1 << 31) == w4.ERANGE
    assert read(plan(), k=P(A + 8)) == w4.EALIGN and read(plan(), v=P(A + 0x8000)) == w4.EALIAS
    assert read(plan(), T=0) == w4.OK
    # nothing there, nothing needed
    assert read(plan(B=0, page_table=None, kv_len=None, cu_rows=None)) == w4.OK


def test_append_errors():
    F = w4.lib().kv_q4_append
    def call(kv=None, r=rope(), k=P(A), ks=256, v=P(A + 0x1000), vs=256, q=None, qs=512, qo=None,
             NH=4, T=4):
        return F(ctypes.byref(kv or plan()), None if r is None else ctypes.byref(r), k, ks, v, vs, q,
                 qs, qo, NH, T, None)
    Q, QO = P(A + 0x8000), P(A + 0x9000)
    assert call(k=None) == w4.ENULL and call(v=None) == w4.ENULL and call(q=Q) == w4.ENULL
    for kw in (dict(ks=252), dict(vs=255), dict(ks=258), dict(T=-1), dict(q=Q, qo=QO, r=None),
               dict(q=Q, qo=QO, NH=0), dict(q=Q, qo=QO, qs=500), dict(q=Q, qo=QO, qs=514),
               dict(r=rope(n_rot=130)), dict(r=rope(mscale=NAN))):
        assert call(**kw) == w4.ESHAPE, kw
    assert call(T=1 << 31) == w4.ERANGE and call(ks=1 << 31) == w4.ERANGE
    assert call(q=Q, qo=QO, NH=1 << 16, qs=1 << 30) == w4.ERANGE
    assert call(k=P(A + 4)) == w4.EALIGN and call(q=P(A + 4), qo=QO) == w4.EALIGN
    assert call(r=rope(inv_freq=A + 4)) == w4.EALIGN
    assert call(q=Q, qo=P(A)) == w4.EALIAS and call(q=Q, qo=Q, qs=516) == w4.EALIAS
    assert call(T=0) == w4.OK and call(kv=plan(B=0)) == w4.OK


def test_attention_errors():
    L = w4.lib()
    S = lambda kv, T, NH: L.attn_q4_workspace_size(ctypes.byref(kv), T, NH)
    assert S(plan(), 4, 4) > 0 and S(plan(), 0, 4) > 0
    assert S(plan(), 4, 3) == 0 and S(plan(), -1, 4) == 0 and S(plan(D=96), 4, 4) == 0
    assert S(plan(), 1 << 30, 4) == 0
    assert L.attn_q4_workspace_size(None, 4, 4) == 0
    # sizes only: the pointers are not looked at
    assert S(plan(k_pages=None, kv_len=None), 4, 4) == S(plan(), 4, 4)
    big = plan(max_pages=4096)
    n = S(big, 4, 4)
    def call(kv=big, q=P(A), qs=512, o=P(A + 0x8000), lse=P(A + 0x9000), T=4, NH=4, scale=0.1,
             window=0, ws=P(A + 0x10000), nb=n):
        return L.attn_q4_forward(ctypes.byref(kv), q, qs, o, lse, T, NH, scale, window, ws, nb, None)
    assert call(q=None) == w4.ENULL and call(o=None) == w4.ENULL and call(ws=None) == w4.ENULL
    for kw in (dict(NH=3), dict(NH=0), dict(T=-1), dict(window=-1), dict(qs=508), dict(qs=514),
               dict(scale=INF), dict(scale=NAN)):
        assert call(**kw) == w4.ESHAPE, kw
    assert call(T=1 << 30) == w4.ERANGE and call(qs=1 << 31) == w4.ERANGE
    assert call(q=P(A + 4)) == w4.EALIGN and call(lse=P(A + 2)) == w4.EALIGN
    assert call(ws=P(A + 8)) == w4.EALIGN
    assert call(o=P(A)) == w4.EALIAS
    assert call(nb=n - 1) == w4.EWORKSPACE
    assert call(T=0) == w4.OK and call(kv=plan(B=0, max_pages=4096)) == w4.OK


def test_attention_refuses_very_large_groups():
    """From 2^16 heads a group on the rows of a tile are not told apart."""
    L = w4.lib()
    kv = plan(max_pages=4096)
    assert kv.NKV == 2
    for NH, rc in ((2 << 16, w4.ERANGE), ((2 << 16) - 2, w4.EWORKSPACE)):
        assert (L.attn_q4_workspace_size(ctypes.byref(kv), 1, NH) == 0) == (rc == w4.ERANGE)
        assert L.attn_q4_forward(ctypes.byref(kv), P(A), NH * 128, P(A + 0x8000), None, 1, NH, 0.1, 0,
                                 P(A + 0x10000), 0, None) == rc


def test_logprobs_errors():
    L = w4.lib()
    S = L.token_logprobs_workspace_size
    assert S(1, 151936, 20) > 0 and S(0, 10, 0) > 0
    assert S(1, 0, 0) == 0 and S(1, 1 << 24, 0) == 0 and S(1, 100, 33) == 0 and S(1, 5, 6) == 0
    assert S(-1, 5, 0) == 0
    n = S(4, 1000, 5)
    def call(x=P(A), st=1000, tg=P(A + 0x4000), lp=P(A + 0x5000), en=P(A + 0x6000),
             ids=P(A + 0x7000), tp=P(A + 0x8000), T=4, V=1000, k=5, ws=P(A + 0x10000), nb=n):
        return L.token_logprobs(x, st, tg, lp, en, ids, tp, T, V, k, ws, nb, None)
    for kw in (dict(x=None), dict(ws=None), dict(tg=None), dict(lp=None), dict(ids=None),
               dict(tp=None)):
        assert call(**kw) == w4.ENULL, kw
    assert call(T=-1) == w4.ESHAPE and call(V=0) == w4.ESHAPE and call(st=999) == w4.ESHAPE
    for kw in (dict(V=1 << 24, st=1 << 24), dict(k=33), dict(k=-1), dict(V=4, k=5),
               dict(st=1 << 39), dict(T=1 << 31)):
        assert call(**kw) == w4.ERANGE, kw
    assert call(x=P(A + 8)) == w4.EALIGN and call(ids=P(A + 0x7002)) == w4.EALIGN
    assert call(nb=n - 1) == w4.EWORKSPACE
    assert call(T=0) == w4.OK


def test_binding_refuses_wrong_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 2, 64)
    pos, f = torch.zeros(4, dtype=torch.int32), torch.zeros(16, dtype=torch.float64)
    with pytest.raises(ValueError):
        w4.rope_rotate(x, pos, f)                                # not on a GPU
    with pytest.raises(ValueError):
        w4.rope_rotate(x.double(), pos, f)
    with pytest.raises(ValueError):
        w4.rope_rotate(x.transpose(1, 2), pos, f)
    with pytest.raises(ValueError):
        w4.rope_rotate(x, pos[:3], f)
    with pytest.raises(ValueError):
        w4.rope_rotate(x, pos, f.float())
    with pytest.raises(ValueError):
        w4.rope_rotate(x, pos, f, layout="other")
    kp, vp = w4.kv_pools(3, 2, 64, device="cpu")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    kv = w4.KVCache(kp, vp, torch.zeros(1, 3, dtype=torch.int32), i32(5), i32(0, 4), 64)
    with pytest.raises(ValueError):
        w4.KVCache(kp, vp, torch.zeros(1, 3, dtype=torch.int32), i32(5, 6), i32(0, 4), 64)
    with pytest.raises(ValueError):
        w4.KVCache(kp[..., :-16], vp, torch.zeros(1, 3, dtype=torch.int32), i32(5), i32(0, 4), 64)
    with pytest.raises(w4.W4A8Error):
        w4.KVCache(kp, vp, torch.zeros(1, 3, dtype=torch.int32), i32(5), i32(0, 4), 96)
    with pytest.raises(ValueError):
        w4.kv_append(kv, x, x[:, :1])
    with pytest.raises(ValueError):
        w4.kv_append(kv, x, x, pos=pos)
    with pytest.raises(ValueError):
        w4.attn_forward(kv, torch.zeros(4, 2, 128), 0.1)
    with pytest.raises(ValueError):
        w4.token_logprobs(torch.zeros(3, 10).t())
    with pytest.raises(ValueError):
        w4.token_logprobs(torch.zeros(3, 10), targets=torch.zeros(3, dtype=torch.int64))


# ------------------------------------------------------------------ the plain forms themselves
def test_plain_rotation_keeps_lengths_and_relative_angles():
    g = np.random.default_rng(1)
    f = ref.frequencies(32)
    q, k = g.standard_normal((1, 1, 40)), g.standard_normal((1, 1, 40))
    for layout in ("half", "interleaved"):
        at = lambda x, p: ref.rotate(x, [p], f, layout)[0, 0]
        assert abs(np.linalg.norm(at(q, 77)) - np.linalg.norm(q)) < 1e-12
        assert abs(at(q, 105) @ at(k, 100) - at(q, 5) @ at(k, 0)) < 1e-12
        assert np.array_equal(at(q, 9)[32:], q[0, 0, 32:])
    x = np.zeros((1, 1, 4))
    x[0, 0, 0] = 1.0
    assert np.allclose(ref.rotate(x, [1], np.array([1.0, 0.5]), "half")[0, 0],
                       [math.cos(1), 0, math.sin(1), 0])
    assert np.allclose(ref.rotate(x, [1], np.array([1.0, 0.5]), "interleaved")[0, 0],
                       [math.cos(1), math.sin(1), 0, 0])


def test_plain_frequencies_by_parts_keep_fast_pairs_and_stretch_slow_ones():
    f = ref.frequencies(128, 10000.0)
    p = ref.frequencies(128, 10000.0, "parts", 8.0, 4096)
    turns = 4096 * f / (2 * math.pi)
    assert np.array_equal(p[turns > 40], f[turns > 40])
    assert np.allclose(p[turns < 0.9] * 8, f[turns < 0.9], rtol=1e-15)
    assert np.all((p <= f) & (p >= f / 8 * (1 - 1e-15)))


def test_plain_tiles_round_trip():
    g = np.random.default_rng(2)
    for fmt, D in (("q4_0", 64), ("q4_sym", 128)):
        x = g.standard_normal((64, D)).astype(np.float32)
        codes, d = ref.codes4(x, fmt)
        for is_k in (True, False):
            pool = g.integers(0, 256, (1, 1, ref.tile_bytes(D, fmt))).astype(np.uint8)
            for t in range(64):
                ref.put(pool, 0, 0, t, codes[t], d[t], fmt, is_k)
            c2, d2 = ref.tile_rows(pool[0, 0], D, fmt, is_k)
            assert np.array_equal(c2, codes) and np.array_equal(d2, d)


def test_plain_logprobs_on_a_known_row():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125]]))
    lp, ent, ids, top, *_ = ref.logprobs(x, [2], 3)
    assert abs(lp[0] - math.log(0.125)) < 1e-15 and abs(ent[0] - 1.75 * math.log(2)) < 1e-15
    assert list(ids[0]) == [0, 1, 2] and abs(top[0, 1] - math.log(0.25)) < 1e-15


def test_plain_quantizers_are_the_oracles_but_for_an_ulp_of_the_scale():
    import oracle
    oracle.build()
    g = np.random.default_rng(3)
    x = (g.standard_normal((400, 64)) * np.exp2(g.integers(-8, 8, (400, 1)))).astype(np.float32)
    raw = np.asarray(oracle.q4_sym_quantize(x)).reshape(400, 2, 20)
    d0 = np.ascontiguousarray(raw[..., :4]).view(np.float32)[..., 0]
    codes, d = ref.codes4(x, "q4_sym")
    assert np.all(np.abs(d - d0) <= np.spacing(d0)) and (d != d0).any() and (d == d0).any()
    pay = np.concatenate([raw[..., 4:] & 15, raw[..., 4:] >> 4], -1)
    assert np.array_equal(codes[d == d0], pay[d == d0])
    for fmt, n, q in (("q4_0", 34, oracle.q8_0_quantize), ("q4_sym", 36, oracle.q8_f32_quantize)):
        raw = np.asarray(q(x)).reshape(400, 2, n)
        d0 = np.ascontiguousarray(raw[..., :n - 32]).view(np.float16 if n == 34 else np.float32)
        v0 = np.ascontiguousarray(raw[..., n - 32:]).view(np.int8).astype(np.float64) * d0
        v = ref.values8(x, fmt).reshape(v0.shape)
        same = (v == v0).all(-1)
        assert same.mean() > (0.99 if n == 34 else 0.2)
        assert np.all(np.abs(v - v0) <= 1.01 * np.abs(d0))
