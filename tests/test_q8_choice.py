"""Which kernel the 8-bit product takes: every one is reached by the sizes that
its GPU tests have, on the 256 compute units of an MI355X."""
import pytest

from tests.kernel_choice import Q8_WAYS, q8_way

# sizes (M, N) for every kernel: rows and channels that end inside tiles, rows of y
# that start 16-byte aligned (N % 4 == 0) and that do not, more row tiles than a
# group of 8 and fewer
SIZES = {
    "few 1x1": [(1, 77), (16, 1000), (1, 40001)],
    "few 1x2": [(2, 32769), (16, 33000)],
    "few 2x1": [(17, 333), (32, 4096)],
    "few 3x1": [(33, 4001), (48, 260)],
    "few 4x1": [(49, 4093), (64, 132)],
    "256x256": [(947, 12291), (2100, 8196)],
    "256x128": [(1030, 4099), (650, 6500), (4500, 1027)],
    "128x128": [(300, 8195), (700, 4100), (1999, 1999)],
    "128x64": [(333, 4099), (947, 2052), (513, 3001)],
    "64x64": [(129, 3001), (65, 5000), (1000, 77)],
}


def test_sizes_are_for_every_kernel():
    assert tuple(SIZES) == Q8_WAYS


@pytest.mark.parametrize("way", Q8_WAYS)
def test_each_kernel_has_its_sizes(way):
    for M, N in SIZES[way]:
        assert q8_way(M, N, 256) == way, (M, N)
