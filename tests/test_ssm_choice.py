"""Which kernels a call of the state space scan takes."""
import pytest

from tests.kernel_choice import ssm_way

SIZES = [1, 2, 7, 8, 9, 16, 48, 63, 64, 65, 128, 500, 947, 1023, 1024, 1025, 3000, 20000]


@pytest.mark.parametrize("B", SIZES)
def test_every_row_is_taken_and_long_sequences_by_chunks(B):
    """Sequences go row by row up to a bound of their length, which is never past
    a chunk (but where there are exactly as many sequences as rows); all that may be
    longer go by chunks: the longest, as many as fit in the call's rows, or all where
    they are not ordered."""
    for T in SIZES:
        w = ssm_way(B, T, 64, 64, 128, 256)
        assert 0 <= w.rows <= (T if T == B else 64)
        longer = min(B, T // (w.rows + 1))
        assert w.chunked == (B if longer and B > 1024 else longer), (B, T, w)


def test_single_tokens_are_one_launch():
    for B in (1, 3, 48, 64, 300, 4000):
        assert ssm_way(B, B, 64, 64, 128, 256)[:3] == (B, True, 0)
    assert ssm_way(1, 8, 64, 64, 128, 256)[:3] == (8, False, 0)


def test_slices():
    """32 columns where there are two workgroups of them for each compute unit."""
    for N, B, NH, P, want in ((128, 4, 64, 64, 32), (128, 3, 64, 64, 16), (128, 1, 256, 64, 32), (128, 1, 255, 64, 16),
                              (128, 1, 256, 80, 32), (128, 1, 256, 48, 16), (64, 1, 1, 64, 32), (256, 64, 64, 64, 16)):
        assert ssm_way(B, 2000 * B, NH, P, N, 256).slice == want, (N, B, NH, P)
