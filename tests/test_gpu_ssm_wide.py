"""The state space scan where a workgroup takes 32 columns of 128 rows of the
state (two workgroups a compute unit), by the library's own choice: a few heads of
many against the recurrence in 64 bits (GPU)."""
import numpy as np
import pytest

from tests import mix_ref as ref
from tests.kernel_choice import ssm_way

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from tests.test_gpu_ssm import Case, whole_numbers

CUS = torch.cuda.get_device_properties(0).multi_processor_count
N = 128


def heads(B, P):
    """The fewest heads that a call of B sequences takes 32 columns for."""
    return -(-2 * CUS // (B * (P // 32)))


def check(c, exact=False):
    B, T, NH, P = len(c.cu) - 1, c.T, c.x.shape[1], c.x.shape[2]
    assert ssm_way(B, T, NH, P, N, CUS).slice == 32
    y, st = c.run()
    some = sorted({0, 1, NH // 2, NH - 1})
    of = lambda a: None if a is None else a[:, some]
    one = lambda a: None if a is None else a[some]
    want, by, new, bs = ref.scan(c.cu, c.src, c.dst, of(c.x), of(c.dt), one(c.A), c.B, c.C, of(c.state), one(c.D), of(c.z),
                                 one(c.bias), c.softplus)
    y, st = y[:, some], st[:, some]
    none = np.isnan(want)
    assert np.all(y[none] == 7.0)
    if exact:
        assert np.array_equal(y[~none], want[~none].astype(np.float32)) and np.array_equal(st, new.astype(np.float32))
    else:
        assert np.all((np.abs(y - want) <= by)[~none]) and np.all(np.abs(st - new) <= bs)


# columns that end with a slice and inside one, one chunk to several
@pytest.mark.parametrize("P", [32, 48, 64, 80])
@pytest.mark.parametrize("lens", [[65], [64, 9], [129], [200, 70, 1, 130]])
def test_wide_slices(P, lens):
    NH = heads(len(lens), P)
    check(whole_numbers(Case([60, P, *lens], lens, N=N, P=P, NH=NH)), exact=True)
    check(Case([61, P, *lens], lens, N=N, P=P, NH=NH))


def test_wide_slices_with_state_in_place_and_rows_of_no_sequence():
    check(Case([62], [70, 0, 150], N=N, P=80, NH=heads(3, 80), lead=5, tail=70, n_slots=3, src=[2, 0, 1], dst=[2, 0, 1]))


def test_values_that_are_not_finite_in_wide_slices():
    NH = heads(2, 48)
    c = Case([63], [100, 100], N=N, P=48, NH=NH, gate=False, n_slots=2, src=[-1] * 2, dst=[0, 1])
    clean, cst = c.run()
    c.x[40, 1, 45] = np.nan
    y, st = c.run()
    hit = np.zeros(clean.shape, bool)
    hit[:100, 1] = True
    assert np.array_equal(y[~hit], clean[~hit]) and np.isnan(y[40:100, 1, 45]).all()
    sh = np.zeros(cst.shape, bool)
    sh[0, 1] = True
    assert np.array_equal(st[~sh], cst[~sh])
