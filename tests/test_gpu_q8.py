"""8-bit rows and their product against the plain forms in 64 bits (GPU).
Codes and scales bit for bit; products within the roundings that their
definition has (tests/mix_ref.py), and exact where those vanish."""
import numpy as np
import pytest

import paper_2606_24031_amd as w4
from tests import mix_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def rng(*seed):
    return np.random.default_rng(seed)


def codes(g, rows, K):
    """Random rows of all int8 values, zeros past K."""
    q = np.zeros((rows, -(-K // 128) * 128), np.int8)
    q[:, :K] = g.integers(-128, 128, (rows, K))
    return q


@pytest.mark.parametrize("rows,K", [(1, 1), (3, 5), (1, 2048), (7, 127), (2, 128), (5, 129), (64, 1541), (9, 4096),
                                    (4, 5000), (2, 16384), (1, 20001), (1, 131071), (300, 64), (33, 8192)])
def test_quantizer_is_its_definition(rows, K):
    g = rng(1, rows, K)
    x = (g.standard_normal((rows, K)) * np.exp2(g.integers(-30, 30, (rows, 1)))).astype(np.float32)
    q, d = w4.q8_row_quantize(dev(x))
    qr, dr = ref.quantize(x)
    assert np.array_equal(d.cpu().numpy(), dr) and np.array_equal(q.cpu().numpy(), qr)


@pytest.mark.parametrize("K", [4, 63, 2048, 9000])
def test_quantizer_special_rows(K):
    """Ties, zeros, subnormals, the ends of fp32, and rows that are not
    finite, beside rows that are."""
    g = rng(2, K)
    x = np.zeros((16, K), np.float32)
    x[0] = np.arange(K) % 255 - 127.0
    x[0, 0], x[1, 0] = 127.0, 127.0                       # scale 1: halves are ties
    x[1, 1:] = (g.integers(-126, 126, K - 1) + 0.5)
    x[3, -1] = 1e-45
    x[4] = g.standard_normal(K) * 1e-39
    x[5] = g.standard_normal(K) * 1e38
    x[5, 0] = np.float32(3.4e38)
    x[6], x[6, K // 2] = 1.0, np.nan
    x[7], x[7, -1] = 1.0, np.inf
    x[8], x[8, 0] = 1.0, -np.inf
    x[9], x[9, -1] = np.nan, 2.0
    x[10:] = g.standard_normal((6, K))
    x[10, 0] = -0.0
    q, d = w4.q8_row_quantize(dev(x))
    qr, dr = ref.quantize(x)
    assert np.array_equal(d.cpu().numpy(), dr, equal_nan=True) and np.array_equal(q.cpu().numpy(), qr)


@pytest.mark.parametrize("K,pad,off", [(200, 40, 0), (201, 0, 0), (202, 7, 1), (256, 16, 4), (2047, 5, 3), (2052, 8, 2)])
def test_quantizer_takes_slices_of_wider_rows(K, pad, off):
    g = rng(3, K)
    wide = g.standard_normal((6, K + pad + off)).astype(np.float32)
    t = dev(wide)[:, off:off + K]
    q, d = w4.q8_row_quantize(t)
    qr, dr = ref.quantize(wide[:, off:off + K])
    assert np.array_equal(d.cpu().numpy(), dr) and np.array_equal(q.cpu().numpy(), qr)


def check(M, N, K, bias, g, out=None):
    xq, wq = codes(g, M, K), codes(g, N, K)
    xd = np.exp2(g.uniform(-8, 2, M)).astype(np.float32)
    wd = np.exp2(g.uniform(-12, -4, N)).astype(np.float32)
    b = g.standard_normal(N).astype(np.float32) if bias else None
    y = w4.q8q8_gemm(dev(xq), dev(xd), dev(wq), dev(wd), bias=dev(b), out=out).cpu().numpy()
    want, bound = ref.product(xq, xd, wq, wd, b)
    bad = ~(np.abs(y - want) <= bound)
    assert not bad.any(), (M, N, K, np.argwhere(bad)[:5], y[bad][:5], want[bad][:5])


# one row to tiles of every kind, rows and channels that end inside a tile,
# one code to long rows
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 48, 64, 65, 100, 128, 129, 200, 257, 300])
@pytest.mark.parametrize("N,K,bias", [(1, 1, True), (16, 128, False), (77, 300, True), (128, 2048, False),
                                      (301, 1541, True), (640, 520, False)])
def test_product(M, N, K, bias):
    check(M, N, K, bias, rng(4, M, N, K))


@pytest.mark.parametrize("M,N,K,bias", [(1, 12288, 2048, False), (3, 40000, 512, True), (1, 5, 131071, False),
                                        (70, 9, 70001, True), (947, 2048, 1024, False), (1030, 4099, 384, True),
                                        (2050, 1000, 640, False), (64, 2048, 4096, True), (5, 2048, 16384, False),
                                        (513, 8200, 256, True)])
def test_product_larger(M, N, K, bias):
    check(M, N, K, bias, rng(5, M, N, K))


@pytest.mark.parametrize("M", [1, 20, 70, 300])
def test_product_largest_sums_are_exact(M):
    """Codes of -128 and 127 throughout, scales of 1: the sums, up to 2^31,
    rounded once."""
    g = rng(6, M)
    K, N = 131071, 20
    xq = np.full((M, K + 1), -128, np.int8)
    wq = np.full((N, K + 1), -128, np.int8)
    wq[1::2] = 127
    xq[:, K], wq[:, K] = 0, 0
    xq[0, ::3] = 5
    y = w4.q8q8_gemm(dev(xq), torch.ones(M, device="cuda"), dev(wq), torch.ones(N, device="cuda")).cpu().numpy()
    s = xq.astype(np.float64) @ wq.astype(np.float64).T
    assert np.array_equal(y, s.astype(np.float32))


@pytest.mark.parametrize("M,N,K", [(1, 100, 256), (40, 256, 640), (200, 77, 384), (300, 520, 1024)])
def test_product_into_slices_of_wider_rows(M, N, K):
    """Nothing but the rows' N channels is written."""
    for pad, off in ((4, 0), (12, 8), (5, 3)):
        wide = torch.full((M, N + pad + off), 7.0, device="cuda")
        check(M, N, K, True, rng(7, M, N, K), out=wide[:, off:off + N])
        assert bool((wide[:, :off] == 7).all()) and bool((wide[:, off + N:] == 7).all())


@pytest.mark.parametrize("M,N,K", [(1, 40, 200), (30, 60, 300), (150, 200, 500)])
def test_codes_past_k_count_only_where_both_are_not_zero(M, N, K):
    g = rng(8, M)
    xq, wq = codes(g, M, K), codes(g, N, K)
    wq2 = wq.copy()
    wq2[:, K:] = g.integers(-128, 128, wq2[:, K:].shape)
    one = lambda n: torch.ones(n, device="cuda")
    a = w4.q8q8_gemm(dev(xq), one(M), dev(wq), one(N))
    assert torch.equal(a, w4.q8q8_gemm(dev(xq), one(M), dev(wq2), one(N)))


@pytest.mark.parametrize("M,N,K", [(3, 50, 200), (40, 64, 256), (200, 300, 700)])
def test_rows_that_are_not_finite_stay_by_themselves(M, N, K):
    g = rng(9, M)
    x, w = g.standard_normal((M, K)).astype(np.float32), g.standard_normal((N, K)).astype(np.float32)
    wq, wd = w4.q8_row_quantize(dev(w))
    clean = w4.q8q8_gemm(*w4.q8_row_quantize(dev(x)), wq, wd).cpu().numpy()
    x[1, 5], x[M - 1, 0] = np.nan, np.inf
    y = w4.q8q8_gemm(*w4.q8_row_quantize(dev(x)), wq, wd).cpu().numpy()
    assert np.isnan(y[[1, M - 1]]).all()
    rest = [m for m in range(M) if m not in (1, M - 1)]
    assert np.array_equal(y[rest], clean[rest])


def test_scales_at_the_ends_of_fp32():
    """The scales' product comes first: a large and a small one do not
    overflow on the way."""
    g = rng(10)
    M, N, K = 20, 70, 300
    xq, wq = codes(g, M, K), codes(g, N, K)
    for a, b in ((1e36, 1e-30), (1e-30, 1e36), (1e-25, 1e-10)):
        xd, wd = np.full(M, a, np.float32), np.full(N, b, np.float32)
        y = w4.q8q8_gemm(dev(xq), dev(xd), dev(wq), dev(wd)).cpu().numpy()
        want, bound = ref.product(xq, xd, wq, wd)
        assert np.all(np.abs(y - want) <= bound + 1e-38)


def test_no_rows():
    w = torch.zeros(8, 128, dtype=torch.int8, device="cuda")
    q, d = w4.q8_row_quantize(torch.zeros(0, 100, device="cuda"))
    assert q.shape == (0, 128)
    assert w4.q8q8_gemm(q, d, w, torch.ones(8, device="cuda")).shape == (0, 8)


@pytest.mark.parametrize("M", [1, 32, 500])
def test_equal_bits_from_call_to_call(M):
    g = rng(11, M)
    N, K = 1000, 2048
    x, w = dev(g.standard_normal((M, K)).astype(np.float32)), dev(g.standard_normal((N, K)).astype(np.float32))
    wq, wd = w4.q8_row_quantize(w)
    y = w4.q8q8_gemm(*w4.q8_row_quantize(x), wq, wd)
    for _ in range(5):
        assert torch.equal(y, w4.q8q8_gemm(*w4.q8_row_quantize(x), wq, wd))
