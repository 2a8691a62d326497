"""Storing into and reading from the paged 4-bit cache (GPU): every byte of
the pools against the oracle's quantizers in the header's layout."""
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


def expect(c, k, v):
    """The pools after storing rows k, v."""
    kp, vp = c.k_pool.copy(), c.v_pool.copy()
    T, NKV, D = k.shape
    kc, kd = ref.codes4(k, c.fmt)
    vc, vd = ref.codes4(v, c.fmt)
    for s in range(len(c.len)):
        for r in range(c.cu[s], c.cu[s + 1]):
            t = int(c.len[s]) - (int(c.cu[s + 1]) - r)
            if t < 0 or t >= c.table.shape[1] * 64:
                continue
            page = c.table[s, t // 64]
            if not 0 <= page < kp.shape[0]:
                continue
            for h in range(NKV):
                i = r * NKV + h
                ref.put(kp, page, h, t % 64, kc[i], kd[i], c.fmt, True)
                ref.put(vp, page, h, t % 64, vc[i], vd[i], c.fmt, False)
    return kp, vp


def pools(kv):
    return kv.tensors[0].cpu().numpy(), kv.tensors[1].cpu().numpy()


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
@pytest.mark.parametrize("lens,rows,NKV,D", [
    ([1], [1], 1, 64), ([64, 65, 130], [1, 1, 1], 2, 128), ([7, 200, 64], [7, 130, 64], 2, 256),
    ([300], [300], 3, 64), ([5, 0, 70, 3], [2, 0, 1, 0], 1, 128)])
def test_append_bytes(lens, rows, NKV, D, fmt):
    g = synth.rng(sum(lens) + D)
    c = attn_cases.random_plan(g, lens, rows, NKV, D, fmt)
    k, v = synth.normal_f32(g, (c.T, NKV, D)), synth.normal_f32(g, (c.T, NKV, D), 0.3)
    k[0, 0, :32] = 0.0                       # a zero block
    v[-1, -1, 32:64] = np.arange(-16, 16)    # ties
    kv = attn_cases.on_gpu(c)
    w4.kv_append(kv, dev(k), dev(v))
    want = expect(c, k, v)
    got = pools(kv)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    ko, vo = w4.kv_read(kv, c.T)
    for o, x in ((ko, k), (vo, v)):
        codes, d = ref.codes4(x, fmt)
        val = ((codes.astype(np.float32) - 8) * d.astype(np.float32)[..., None]).reshape(x.shape)
        assert np.array_equal(o.cpu().numpy(), val)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n", [128, 32, 58])
def test_append_rotates_keys_and_queries_from_one_projection(layout, n):
    """q, k, v as slices of one row; the stored key is the block of the key
    rotated in fp64 and rounded once."""
    NH, NKV, D = 6, 2, 128
    g = synth.rng(n)
    c = attn_cases.random_plan(g, [70, 33, 640], [3, 33, 600], NKV, D, "q4_0")
    qkv = synth.normal_f32(g, (c.T, NH + 2 * NKV, D))
    pos = np.concatenate([np.arange(a - b, a) for a, b in zip([70, 33, 640], [3, 33, 600])]).astype(np.int32)
    f = ref.frequencies(n)
    kv, b = attn_cases.on_gpu(c), dev(qkv)
    qr = w4.kv_append(kv, b[:, NH:NH + NKV], b[:, NH + NKV:], pos=dev(pos), inv_freq=dev(f),
                      layout=layout, q=b[:, :NH])
    # fp64 on both sides, rounded to fp32 once: equal but for a value on a rounding border
    k = ref.rotate(qkv[:, NH:NH + NKV], pos, f, layout).astype(np.float32)
    want = expect(c, k, qkv[:, NH + NKV:])
    got = pools(kv)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    q64 = ref.rotate(qkv[:, :NH], pos, f, layout)
    assert np.all(np.abs(qr.cpu().numpy() - q64) <= 2.0 ** -24 * np.abs(q64) + 2.0 ** -36)
    assert torch.equal(b, dev(qkv))
    # q rotated in place when it is contiguous
    q = dev(qkv[:, :NH])
    w4.kv_append(kv, b[:, NH:NH + NKV], b[:, NH + NKV:], pos=dev(pos), inv_freq=dev(f),
                 layout=layout, q=q, q_out=q)
    assert torch.equal(q, qr)


def test_rows_without_a_place_are_dropped():
    """Tokens before 0 and past the table, absent pages (-1, past the pool),
    rows of no sequence: nothing but the present rows' bytes changes, and
    reading gives zeros there, and leaves rows of no sequence as they were."""
    NKV, D = 2, 64
    g = synth.rng(77)
    c = attn_cases.random_plan(g, [2, 200, 130, 90], [5, 3, 130, 2], NKV, D, "q4_0", capacity=4)
    c.table[1, 3] = -1                       # the page of tokens 192 .. 199
    c.table[2, 1] = c.k_pool.shape[0]        # tokens 64 .. 127
    c.len[3] = 257                           # 256 lies past 4 pages
    T = c.T + 3                              # three rows behind the last sequence
    k, v = synth.normal_f32(g, (T, NKV, D)), synth.normal_f32(g, (T, NKV, D))
    kv = attn_cases.on_gpu(c)
    w4.kv_append(kv, dev(k), dev(v))
    want = expect(c, k, v)
    got = pools(kv)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    ko = torch.full((T, NKV, D), 5.0, device="cuda")
    ko, vo = w4.kv_read(kv, T, k_out=ko)
    ko = ko.cpu().numpy()
    assert np.all(ko[c.T:] == 5.0)
    assert np.all(ko[:3] == 0.0) and np.all(ko[3:5] != 5.0)          # tokens -3, -2, -1 | 0, 1
    assert np.all(ko[5:8] == 0.0)
    assert np.all(ko[8 + 64:8 + 128] == 0.0) and np.any(ko[8 + 128:8 + 130] != 0.0)


@pytest.mark.parametrize("B", [63, 64, 65, 200, 4200])
def test_many_sequences(B):
    """The row's sequence is found by 64 entries at a time: some sequences
    without rows, one row in most."""
    g = synth.rng(B)
    rows = (g.random(B) < 0.7).astype(int)
    rows[-1] = 2
    lens = [int(x) for x in g.integers(2, 60, B)]
    c = attn_cases.random_plan(g, lens, rows, 1, 64, "q4_0", spare=0)
    k, v = synth.normal_f32(g, (c.T, 1, 64)), synth.normal_f32(g, (c.T, 1, 64))
    kv = attn_cases.on_gpu(c)
    w4.kv_append(kv, dev(k), dev(v))
    want = expect(c, k, v)
    got = pools(kv)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def test_no_sequences_still_rotates_queries():
    kp, vp = w4.kv_pools(2, 1, 64)
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    kv = w4.KVCache(kp, vp, torch.empty(0, 2, dtype=torch.int32, device="cuda"), e,
                    torch.zeros(1, dtype=torch.int32, device="cuda"), 64)
    g = synth.rng(3)
    x, q = synth.normal_f32(g, (2, 1, 64)), synth.normal_f32(g, (2, 3, 64))
    pos, f = np.array([4, 9], np.int32), ref.frequencies(64)
    before = kp.clone()
    r = w4.kv_append(kv, dev(x), dev(x), pos=dev(pos), inv_freq=dev(f), q=dev(q))
    assert np.allclose(r.cpu().numpy(), ref.rotate(q, pos, f), atol=1e-6)
    assert torch.equal(kp, before)


@pytest.mark.parametrize("layout,n", [("half", 128), ("half", 58), ("interleaved", 64), ("interleaved", 58)])
@pytest.mark.parametrize("T", [1, 3, 1100])
def test_queries_rotated_in_place(T, layout, n):
    """q_out as q itself: the bits of a call with a buffer of its own, a row on
    one workgroup and on several."""
    NH, NKV, D = 24, 1, 128
    g = synth.rng(T + n)
    c = attn_cases.random_plan(g, [T], [T], NKV, D, "q4_0")
    kv = attn_cases.on_gpu(c)
    q, k, v = (dev(synth.normal_f32(g, (T, h, D))) for h in (NH, NKV, NKV))
    pos, f = torch.arange(T, dtype=torch.int32, device="cuda"), w4.rope_frequencies(n)
    want = w4.kv_append(kv, k, v, pos=pos, inv_freq=f, layout=layout, q=q)
    assert torch.equal(want, w4.rope_rotate(q, pos, f, layout))
    pages = [t.clone() for t in kv.tensors[:2]]
    got = w4.kv_append(kv, k, v, pos=pos, inv_freq=f, layout=layout, q=q, q_out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want)
    assert all(torch.equal(a, b) for a, b in zip(pages, kv.tensors[:2]))
