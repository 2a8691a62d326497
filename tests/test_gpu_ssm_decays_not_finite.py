"""Decays of the state space scan that are not finite: the same answer row by
row and chunk by chunk (GPU)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from tests.test_gpu_ssm import Case, whole_numbers


# (short ones go row by row, others by chunks of 64 rows)
@pytest.mark.parametrize("n", [1, 8, 9, 64, 200])
def test_a_head_whose_decay_is_nan_is_nan(n):
    """As the recurrence has it; the other heads' bits are theirs."""
    c = Case([40, n], [n, n], NH=3, n_slots=2, src=[-1, 1], dst=[0, 1])
    clean, cst = c.run()
    c.A[1] = np.nan
    y, st = c.run()
    rest = [0, 2]
    assert np.isnan(y[:, 1]).all() and np.isnan(st[:, 1]).all()
    assert np.array_equal(y[:, rest], clean[:, rest]) and np.array_equal(st[:, rest], cst[:, rest])


@pytest.mark.parametrize("n", [8, 150])
def test_no_step_of_an_infinite_decay_is_nan(n):
    """0 times infinity, from that row (of chunks: from its chunk) on."""
    c = Case([41, n], [n], NH=2, softplus=False, bias=False, n_slots=1, src=[-1], dst=[0])
    clean, cst = c.run()
    c.A[1], c.dt[n // 2, 1] = -np.inf, 0.0
    y, st = c.run()
    assert np.isnan(y[n // 2:, 1]).all() and np.isnan(st[0, 1]).all()
    assert np.array_equal(y[:, 0], clean[:, 0]) and np.array_equal(st[0, 0], cst[0, 0])


@pytest.mark.parametrize("n", [8, 150])
def test_an_infinite_decay_forgets(n):
    whole_numbers(Case([42, n], [n]), keep=-np.inf).check(exact=True)
