"""Attention over the paged 4-bit cache against fp64 (GPU).  Tolerances:
attn_ref.attention_bounds counts the roundings per element."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from paper_2606_24031_amd import synth
from tests import attn_cases, attn_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

REL = []     # (case, largest error over its bound)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def check(c, q, scale, window=0, got=None, what=""):
    if got is None:
        got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), scale, window)
    r = ref.attention(c, q, scale, window)
    bo, bl = ref.attention_bounds(r)
    o, l = got[0].cpu().numpy().astype(np.float64), got[1].cpu().numpy().astype(np.float64)
    assert np.isfinite(o).all(), what
    eo = np.abs(o - r.out) / bo
    assert np.array_equal(np.isneginf(l), np.isneginf(r.lse)), what
    fin = np.isfinite(r.lse)
    el = (np.abs(l - r.lse)[fin] / bl[fin]) if fin.any() else np.zeros(1)
    rel = np.linalg.norm(o - r.out) / max(np.linalg.norm(r.out), 1e-300)
    REL.append((what, float(eo.max()), float(el.max())))
    print(f"attn {what}: error / bound {eo.max():.3g}, lse {el.max():.3g}; relative {rel:.3g}", flush=True)
    assert eo.max() <= 1.0 and el.max() <= 1.0, what
    return r


def case(seed, lens, rows, NH, NKV, D, fmt, **kw):
    g = synth.rng(seed)
    c = attn_cases.random_plan(g, lens, rows, NKV, D, fmt, **kw)
    return c, 2.0 * synth.normal_f32(g, (c.T, NH, D))


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens,rows,NH,NKV", [
    ([1], [1], 1, 1),                                # one key
    ([64], [1], 8, 1), ([65], [1], 4, 2),            # a whole page, one key past it
    ([948], [1], 16, 2),                             # four waves of pages, one run or two
    ([3, 700, 1, 257], [1, 1, 1, 1], 6, 2),          # ragged, three heads a group
])
def test_decode(lens, rows, NH, NKV, D, fmt):
    c, q = case(D + sum(lens), lens, rows, NH, NKV, D, fmt)
    check(c, q, D ** -0.5, what=f"decode {lens} {NH}/{NKV} D={D} {fmt}")


@pytest.mark.parametrize("D,fmt", [(64, "q4_sym"), (128, "q4_0"), (256, "q4_0"), (256, "q4_sym")])
@pytest.mark.parametrize("lens,rows,NH,NKV", [
    ([5], [5], 4, 1), ([16, 40], [16, 7], 2, 2), ([130, 64], [130, 64], 4, 2),
    ([300, 200, 90], [3, 33, 90], 12, 2),            # tiles that end inside a token's heads
])
def test_prompt_rows(lens, rows, NH, NKV, D, fmt):
    c, q = case(D + sum(lens), lens, rows, NH, NKV, D, fmt)
    check(c, q, D ** -0.5, what=f"prompt {lens} {NH}/{NKV} D={D} {fmt}")


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 200, 10 ** 9])
def test_window(window):
    c, q = case(window % 97, [333, 64, 500], [5, 64, 1], 4, 2, 64, "q4_0")
    check(c, q, 0.125, window, what=f"window {window}")


def test_a_window_wider_than_any_sequence():
    c, q = case(3, [4, 333], [9, 5], 4, 2, 64, "q4_0")      # with rows before token 0
    kv = attn_cases.on_gpu(c)
    want = w4.attn_forward(kv, dev(q), 0.125)
    for window in (2 ** 31 - 1, 2 ** 31, 2 ** 63 - 1):
        got = w4.attn_forward(kv, dev(q), 0.125, window)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), window


@pytest.mark.parametrize("D,NH,NKV,lens,rows", [
    (128, 8, 1, [20000], [1]), (256, 16, 2, [9000], [2]), (64, 2, 2, [15000, 40, 7000], [1, 1, 3]),
    (128, 16, 1, [6000, 2500], [4, 1])])
def test_long_contexts_split_into_runs(D, NH, NKV, lens, rows):
    """Long enough that sequences fall into several runs, next to some that do
    not, with 16- and 32-row tiles."""
    c, q = case(D + lens[0], lens, rows, NH, NKV, D, "q4_0")
    check(c, q, D ** -0.5, what=f"long {lens} D={D}")
    if len(lens) == 1:
        check(c, q, D ** -0.5, 5000, what=f"long, window, {lens} D={D}")


def test_more_sequences_than_a_wave_looks_at_once():
    g = synth.rng(4)
    lens = [int(x) for x in g.integers(1, 150, 150)]
    rows = [min(n, int(x)) for n, x in zip(lens, g.integers(0, 3, 150))]
    c, q = case(8, lens, rows, 2, 1, 64, "q4_0")
    check(c, q, 0.125, what="150 sequences")
    lens[70], rows[70], lens[140] = 9000, 1, 5000
    c, q = case(9, lens, rows, 2, 1, 64, "q4_0")
    check(c, q, 0.125, what="150 sequences, two of them long")


def test_rows_that_see_nothing():
    """No tokens, tokens before the first, absent pages: zeros and -infinity;
    rows of no sequence keep their contents."""
    c, q = case(31, [0, 3, 70, 200], [2, 5, 1, 2], 4, 2, 64, "q4_0")
    c.table[2, :] = -1
    c.table[3, 1:] = c.k_pool.shape[0] + 5           # only the first page is there
    T = c.T + 2
    q = np.concatenate([q, np.full((2, 4, 64), np.nan, np.float32)])
    out, lse = torch.full((T, 4, 64), 7.0, device="cuda"), torch.full((T, 4), 7.0, device="cuda")
    w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125, out=out, lse=lse)
    assert bool((out[c.T:] == 7.0).all()) and bool((lse[c.T:] == 7.0).all())
    r = check(c, q[:c.T], 0.125, got=(out[:c.T], lse[:c.T]), what="nothing seen")
    assert list(r.keys) == [0, 0, 0, 0, 1, 2, 3, 0, 64, 64]
    # a window that lies on absent pages only
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125, window=60)
    assert bool((got[0][8:10] == 0).all()) and bool(torch.isneginf(got[1][8:10]).all())


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
def test_what_a_row_does_not_see_does_not_enter_it(fmt):
    """NaN, infinite and huge scales of keys outside a row's window and after
    it (another row of the tile sees them); that other row gets NaN only."""
    D, NH = 64, 2
    c, q = case(6, [130], [6], NH, 1, D, fmt)
    clean = ref.attention(c, q, 0.125, 40)
    ft = np.float16 if fmt == "q4_0" else np.float32
    at = lambda t: (t % 16) // 4 * 16 + t // 16 * 4 + t % 4
    for pool in (c.k_pool, c.v_pool):
        for tok, x in ((129, np.nan), (128, np.inf), (20, np.nan), (84, -np.inf), (3, 6e4)):
            sc = pool[c.table[0, tok // 64], 0, D // 32 * 1024:].view(ft)
            sc[at(tok % 64)] = x
            sc[64 + at(tok % 64)] = x
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.125, 40)
    o = got[0].cpu().numpy()
    # rows are tokens 124 .. 129: the first four see 85 .. 127 at most
    bo, bl = ref.attention_bounds(clean)
    assert np.all(np.abs(o[:4] - clean.out[:4]) <= bo[:4])
    assert np.all(np.abs(got[1].cpu().numpy()[:4] - clean.lse[:4]) <= bl[:4])
    assert not np.isfinite(o[5]).any()


@pytest.mark.parametrize("scale", [0.0, -0.125, 3.0])
def test_scales_of_the_scores(scale):
    c, q = case(12, [150, 300], [1, 20], 4, 2, 64, "q4_0")
    check(c, q, scale, what=f"scale {scale}")


@pytest.mark.parametrize("fmt,sizes", [("q4_0", (2.0 ** -12, 2.0 ** 10)), ("q4_sym", (2.0 ** -100, 2.0 ** 90))])
def test_value_scales_of_any_size(fmt, sizes):
    """Value scales that grow and shrink along the sequence by 2^12 within a
    tile, and all tiny or all huge: the halves' common power of two follows."""
    for i, base in enumerate((1.0,) + sizes):
        c, q = case(40 + i, [700], [1], 4, 1, 128, fmt)
        ft = np.float16 if fmt == "q4_0" else np.float32
        step = np.exp2(np.linspace(-6, 6, 11))
        for j, p in enumerate(c.table[0, :11]):
            sc = c.v_pool[p][:, 4 * 1024:].view(ft)
            with np.errstate(over="ignore"):
                sc[:] = (sc.astype(np.float64) * base * step[j * 7 % 11]).astype(ft)
        check(c, q, 128 ** -0.5, what=f"value scales x {base:.2g} {fmt}")


def test_strided_queries_equal_contiguous_ones():
    c, q = case(15, [90, 200], [3, 2], 6, 2, 128, "q4_0")
    kv = attn_cases.on_gpu(c)
    a = w4.attn_forward(kv, dev(q), 0.1)
    buf = torch.full((c.T, 10, 128), float("nan"), device="cuda")
    buf[:, 2:8] = dev(q)
    b = w4.attn_forward(kv, buf[:, 2:8], 0.1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    d = w4.attn_forward(kv, dev(q), 0.1, want_lse=False)
    assert d[1] is None and torch.equal(a[0], d[0])


def test_sequences_share_a_prefix():
    """Two tables that name the same pages give what separate copies give."""
    c, q = case(16, [256, 256, 200], [1, 1, 1], 4, 2, 64, "q4_0")
    c.table[1, :3] = c.table[0, :3]
    check(c, q, 0.125, what="shared pages")


def test_equal_bits_each_time_and_whatever_the_others_hold():
    c, q = case(17, [5000, 900, 20], [1, 9, 20], 8, 2, 128, "q4_0")
    kv = attn_cases.on_gpu(c)
    a = w4.attn_forward(kv, dev(q), 0.1)
    for _ in range(3):
        b = w4.attn_forward(kv, dev(q), 0.1)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.k_pool[c.table[1, :15]] ^= 0x33
    q2 = q.copy()
    q2[1:10] *= -1
    b = w4.attn_forward(attn_cases.on_gpu(c), dev(q2), 0.1)
    assert torch.equal(a[0][0], b[0][0]) and torch.equal(a[0][10:], b[0][10:])
    assert not torch.equal(a[0][1:10], b[0][1:10])


def test_one_workspace_for_calls_of_several_shapes():
    """A workspace large enough for all serves calls of any shape in turn, on
    either way of joining runs; its arrival counters are zero after each."""
    calls = [case(50, [9000], [1], 8, 1, 256, "q4_0"), case(51, [5000] + [100] * 39, [1] * 40, 4, 1, 64, "q4_0"),
             case(52, [900, 3000], [4, 2], 8, 2, 128, "q4_sym"), case(53, [70], [70], 2, 1, 64, "q4_0")]
    kvs = [attn_cases.on_gpu(c) for c, _ in calls]
    size = max(w4.attn_workspace(kv, c.T, q.shape[1]).numel() for kv, (c, q) in zip(kvs, calls))
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for i in (0, 1, 2, 3, 1, 0, 2):
        c, q = calls[i]
        check(c, q, 0.1, got=w4.attn_forward(kvs[i], dev(q), 0.1, workspace=ws), what=f"shared workspace, call {i}")
        assert not bool(ws[:12288].any())


def test_empty_calls():
    c, q = case(18, [10], [1], 2, 1, 64, "q4_0")
    kv = attn_cases.on_gpu(c)
    o, l = w4.attn_forward(kv, dev(q[:0]), 0.1)
    assert o.shape == (0, 2, 64) and l.shape == (0, 2)


@pytest.mark.parametrize("rows", [1, 30])
def test_a_pool_without_pages(rows):
    """No page is present: rows give zeros and -infinity, stores go nowhere."""
    D, fmt = 64, "q4_0"
    kp, vp = w4.kv_pools(0, 2, D, fmt)
    i32 = lambda a: dev(np.array(a, np.int32))
    kv = w4.KVCache(kp, vp, i32([[0, 1], [-1, 7]]), i32([100, 40]), i32([0, rows, rows + 1]), D, fmt)
    T = rows + 1
    q = torch.randn(T, 4, D, device="cuda")
    out, lse = w4.attn_forward(kv, q, 0.125)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
    w4.kv_append(kv, q[:, :2].contiguous(), q[:, 2:].contiguous())
    k, v = w4.kv_read(kv, T)
    assert bool((k == 0).all()) and bool((v == 0).all())
    # tables without columns
    kv = w4.KVCache(kp, vp, torch.empty(2, 0, dtype=torch.int32, device="cuda"), i32([100, 40]),
                    i32([0, rows, rows + 1]), D, fmt)
    out, lse = w4.attn_forward(kv, q, 0.125)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
def test_rows_without_keys_at_a_large_scale(fmt):
    # rows before token 0 beside rows that see keys, with a scale at which the
    # lowest running maximum times it would overflow
    c, q = case(77, [5, 40], [9, 60], 4, 2, 64, fmt)
    r = check(c, q, 20.0, what=f"rows before token 0 at scale 20, {fmt}")
    assert np.isneginf(r.lse).any() and np.isfinite(r.lse).any()


def test_a_workspace_of_its_own_on_another_stream():
    """Without a workspace the call's own is zero-filled on its stream, not
    behind the current stream's work."""
    c, q = case(31, [700, 90], [3, 2], 8, 2, 64, "q4_0")
    kv, qd = attn_cases.on_gpu(c), dev(q)
    want = w4.attn_forward(kv, qd, 0.125)
    n = w4.attn_workspace(kv, c.T, 8).numel()
    st, out, lse = torch.cuda.Stream(), torch.empty_like(want[0]), torch.empty_like(want[1])
    x = torch.ones(4096, 4096, device="cuda")
    for _ in range(3):
        dirty = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        del dirty
        st.wait_stream(torch.cuda.current_stream())
        for _ in range(20):
            x = torch.tanh(x)                     # the current stream is busy
        w4.attn_forward(kv, qd, 0.125, out=out, lse=lse, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("fmt", ["q4_0", "q4_sym"])
def test_a_prompt_and_what_its_rows_do_not_see(fmt):
    """NaN and infinite scales of a few keys: rows that do not see them (others
    of their tile do) keep their results."""
    D, NH = 128, 12
    c, q = case(7, [1300], [1300], NH, 1, D, fmt)
    clean = ref.attention(c, q, 0.09, 100)
    ft = np.float16 if fmt == "q4_0" else np.float32
    at = lambda t: (t % 16) // 4 * 16 + t // 16 * 4 + t % 4
    bad = {400: np.nan, 801: np.inf, 1190: -np.inf}
    for pool in (c.k_pool, c.v_pool):
        for tok, x in bad.items():
            sc = pool[c.table[0, tok // 64], 0, D // 32 * 1024:].view(ft)
            sc[at(tok % 64)] = x
            sc[3 * 64 + at(tok % 64)] = x
    got = w4.attn_forward(attn_cases.on_gpu(c), dev(q), 0.09, 100)
    o, l = got[0].cpu().numpy(), got[1].cpu().numpy()
    t = np.arange(c.T)
    see = np.any([(t >= k) & (t - 100 < k) for k in bad], axis=0)
    assert see.sum() == 300
    bo, bl = ref.attention_bounds(clean)
    assert np.all(np.abs(o[~see] - clean.out[~see]) <= bo[~see])
    assert np.all(np.abs(l[~see] - clean.lse[~see]) <= bl[~see])
    # only values bad: scores are as they were, and the other columns too
    c2, _ = case(7, [1300], [1300], NH, 1, D, fmt)
    for tok, x in bad.items():
        sc = c2.v_pool[c2.table[0, tok // 64], 0, D // 32 * 1024:].view(ft)
        sc[at(tok % 64)] = x
    got = w4.attn_forward(attn_cases.on_gpu(c2), dev(q), 0.09, 100)
    o, l = got[0].cpu().numpy(), got[1].cpu().numpy()
    assert np.all(np.abs(l - clean.lse) <= bl)
    assert np.all(np.abs(o[~see] - clean.out[~see]) <= bo[~see])
    assert np.all(np.abs(o[see][..., 32:] - clean.out[see][..., 32:]) <= bo[see][..., 32:])
    assert not np.isfinite(o[see][..., :32]).any()


@pytest.mark.parametrize("D,fmt,lens,rows,NH,NKV,window", [
    (64, "q4_0", [500], [500], 66, 2, 0),            # 33 heads a group: tiles end inside a token's
    (128, "q4_sym", [500], [500], 66, 2, 0),
    (256, "q4_0", [270, 30], [260, 7], 126, 2, 0),
    (128, "q4_0", [321, 700], [321, 191], 64, 1, 90),
    (64, "q4_sym", [3, 600, 0], [40, 470, 2], 64, 1, 0),   # rows before token 0, no tokens
    (256, "q4_0", [300], [300], 16, 2, 0), (256, "q4_sym", [70, 600], [70, 200], 16, 1, 100),
])
def test_prompts_of_many_rows(D, fmt, lens, rows, NH, NKV, window):
    """The tiles of large calls: 32 rows, and 16 of 256 columns (the last two)."""
    c, q = case(D + sum(lens), lens, rows, NH, NKV, D, fmt)
    check(c, q, D ** -0.5, window, what=f"many rows {lens} {NH}/{NKV} D={D} {fmt} window {window}")


@pytest.mark.parametrize("D,lens,rows", [(256, [4000], [1]), (64, [9000, 5], [1, 1]), (128, [2500, 3100], [2, 1])])
def test_joins_by_a_launch_and_without(D, lens, rows):
    """Sequences whose runs the last workgroups join in one call and a second
    launch in another (more pages in the plan's tables): the same results."""
    c, q = case(D + len(lens), lens, rows, 4, 2, D, "q4_0")
    check(c, q, D ** -0.5, what=f"joins {lens} D={D}")
    wide = attn_cases.random_plan(synth.rng(1), lens, rows, 2, D, "q4_0", capacity=700)
    wide.k_pool, wide.v_pool = c.k_pool, c.v_pool
    wide.table[:, :c.table.shape[1]] = c.table
    wide.table[:, c.table.shape[1]:] = -1
    check(wide, q, D ** -0.5, what=f"joins, wide tables, {lens} D={D}")
