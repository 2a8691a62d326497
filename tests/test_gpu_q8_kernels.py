"""Every kernel of the 8-bit product at its own sizes, by the library's own
choice, against the plain form in 64 bits (GPU)."""
import pytest

from tests.kernel_choice import q8_way
from tests.test_q8_choice import SIZES

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from tests.test_gpu_q8 import check, rng

CUS = torch.cuda.get_device_properties(0).multi_processor_count


# (stages of 64 codes: 2, as many as a ring of 4 has, more, and many)
@pytest.mark.parametrize("K,bias", [(100, True), (256, False), (300, True), (1541, False)])
@pytest.mark.parametrize("way,M,N", [(w, *s) for w in SIZES for s in SIZES[w]])
def test_kernel(way, M, N, K, bias):
    assert q8_way(M, N, CUS) == way
    check(M, N, K, bias, rng(20, M, N, K))


@pytest.mark.parametrize("way", [w for w in SIZES if "few" not in w])
def test_tiles_into_slices_of_wider_rows(way):
    """Nothing but the rows' N channels is written, with rows that start 16-byte
    aligned and others."""
    M, N = SIZES[way][0]
    for pad, off in ((16 - N % 4, 8), (5 + N % 2, 3)):
        wide = torch.full((M, off + N + pad), 7.0, device="cuda")
        check(M, N, 300, True, rng(21, M, N, pad), out=wide[:, off:off + N])
        assert bool((wide[:, :off] == 7).all()) and bool((wide[:, off + N:] == 7).all())
