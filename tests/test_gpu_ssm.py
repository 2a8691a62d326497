"""The selective state space scan against the recurrence in 64 bits (GPU):
within the bounds of tests/mix_ref.py, and bit for bit where every sum is a
small whole number."""
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


def i32(a):
    return None if a is None else dev(np.asarray(a, np.int32))


class Case:
    def __init__(self, seed, lens, NH=2, P=64, N=64, NG=1, gate=True, D=True, bias=True, softplus=True, lead=0, tail=0,
                 n_slots=None, src=None, dst=None):
        g = self.g = np.random.default_rng(seed)
        f = lambda *s: g.standard_normal(s).astype(np.float32)
        self.cu = lead + np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        T = self.T = int(self.cu[-1]) + tail
        self.n_slots = 2 * len(lens) if n_slots is None else n_slots
        slots = g.permutation(max(self.n_slots, 2 * len(lens)))
        self.src = slots[:len(lens)] if src is None else np.asarray(src)
        self.dst = slots[len(lens):2 * len(lens)] if dst is None else np.asarray(dst)
        step = np.exp(g.uniform(np.log(1e-3), np.log(0.1), NH))
        self.x, self.B, self.C = f(T, NH, P), f(T, NG, N), f(T, NG, N)
        self.z = f(T, NH, P) if gate else None
        self.dt = 0.5 * f(T, NH) if softplus else (step * g.uniform(0.5, 2, (T, NH))).astype(np.float32)
        self.bias = (step + np.log(-np.expm1(-step))).astype(np.float32) if bias else None
        if softplus and not bias:
            self.dt -= 3
        if bias and not softplus:
            self.bias = (0.01 * g.random(NH)).astype(np.float32)
        self.A = -g.uniform(1, 16, NH).astype(np.float32)
        self.D = f(NH) if D else None
        self.state = f(self.n_slots, NH, N, P)
        self.softplus = softplus

    def run(self, rows=None, out=None, workspace=None, stream=None):
        T = self.T if rows is None else rows
        plan = w4.SeqPlan(i32(self.cu), self.n_slots, src=i32(self.src), dst=i32(self.dst))
        st = dev(self.state)
        if out is None:
            out = torch.full(self.x[:T].shape, 7.0, device="cuda")
        d = lambda a: None if a is None else dev(a[:T])
        w4.ssm_scan(plan, d(self.x), d(self.dt), dev(self.A), d(self.B), d(self.C), st if self.n_slots else None,
                    D=dev(self.D), z=d(self.z), dt_bias=dev(self.bias), softplus=self.softplus, out=out,
                    workspace=workspace)
        return out.cpu().numpy(), st.cpu().numpy()

    def check(self, rows=None, exact=False):
        y, st = self.run(rows)
        T = self.T if rows is None else rows
        c = lambda a: None if a is None else a[:T]
        want, by, new, bs = ref.scan(self.cu, self.src, self.dst, self.x[:T], self.dt[:T], self.A, self.B[:T],
                                     self.C[:T], self.state, self.D, c(self.z), self.bias, self.softplus)
        none = np.isnan(want)
        assert np.all(y[none] == 7.0), "rows of no sequence"
        if exact:                # (rounded to fp32: 64 bits hold what is left of a decay of exp(-200))
            f32 = lambda a: a.astype(np.float32)
            assert np.array_equal(y[~none], f32(want[~none])) and np.array_equal(st, f32(new))
            return
        ey, es = np.abs(y - want)[~none] / by[~none], np.abs(st - new) / bs
        print(f"max err/bound: output {ey.max(initial=0):.3g}, state {es.max(initial=0):.3g}", flush=True)
        assert np.all(ey <= 1), np.argwhere(~none & ~(np.abs(y - want) <= by))[:5]
        assert np.all(es <= 1), np.argwhere(~(es <= 1))[:5]


# one row (and up to 8: row by row), the smallest chunk, whole chunks, rows past
@pytest.mark.parametrize("n", [1, 2, 8, 9, 63, 64, 65, 128, 200, 321])
@pytest.mark.parametrize("N,P", [(64, 64), (128, 64), (256, 32), (64, 16), (128, 48), (128, 128)])
def test_lengths(n, N, P):
    Case([1, n, N, P], [n], N=N, P=P).check()


@pytest.mark.parametrize("NH,NG", [(1, 1), (4, 2), (6, 3), (5, 5), (8, 1)])
def test_heads_and_groups(NH, NG):
    Case([2, NH, NG], [70, 3], NH=NH, NG=NG, N=128, P=16).check()


@pytest.mark.parametrize("gate,D,bias,softplus", [(False, False, False, False), (True, False, False, True),
                                                  (False, True, True, False), (False, False, True, True)])
@pytest.mark.parametrize("n", [3, 90])
def test_options(gate, D, bias, softplus, n):
    Case([3, n], [n], gate=gate, D=D, bias=bias, softplus=softplus).check()


@pytest.mark.parametrize("lens", [[1] * 9, [4, 4, 4, 4], [1, 70, 1, 9, 0, 130, 8], [0, 0, 65, 0], [12, 1, 1, 64, 64]])
@pytest.mark.parametrize("N,P", [(64, 32), (128, 64), (256, 16)])
def test_ragged_batches(lens, N, P):
    Case([4, N, *lens], lens, N=N, P=P).check()


def test_rows_of_no_sequence_are_left():
    Case([5], [70, 0, 5], lead=6, tail=70).check()
    Case([5], [1, 1], lead=2, tail=1).check()


@pytest.mark.parametrize("rows", [1, 30, 64, 70, 72, 90, 140])
def test_calls_with_fewer_rows_than_the_plan(rows):
    Case([6, rows], [70, 2, 80]).check(rows=rows)


@pytest.mark.parametrize("lens", [[1, 3, 2], [100, 64, 9]])
def test_state_in_place(lens):
    Case([7, *lens], lens, n_slots=3, src=[2, 0, 1], dst=[2, 0, 1]).check()


def test_absent_slots_begin_with_zeros_and_keep_nothing():
    Case([8], [70, 8, 90, 2], n_slots=4, src=[-1, 1, 4, 2], dst=[0, -1, 3, 1 << 30]).check()


def test_no_slots_at_all():
    c = Case([9], [70, 20, 3], n_slots=0, src=[0, -1, 0], dst=[0, 1, 2])
    c.state = np.zeros((0, 2, 64, 64), np.float32)
    c.check()


def test_several_sequences_read_one_slot():
    Case([10], [70, 20, 3], n_slots=5, src=[1, 1, 1], dst=[0, 2, 4]).check()


def test_default_slots():
    c = Case([11], [70, 20, 3], n_slots=3, src=[0, 1, 2], dst=[0, 1, 2])
    want = c.run()
    st = dev(c.state)
    y = w4.ssm_scan(w4.SeqPlan(i32(c.cu), 3), dev(c.x), dev(c.dt), dev(c.A), dev(c.B), dev(c.C), st, D=dev(c.D),
                    z=dev(c.z), dt_bias=dev(c.bias))
    assert np.array_equal(y.cpu().numpy(), want[0]) and np.array_equal(st.cpu().numpy(), want[1])


def test_strided_rows():
    """x, B and C of one tensor's rows, z and dt of another's, into wider rows."""
    c = Case([12], [70, 3, 9], NH=4, NG=2, N=64, P=32)
    want = c.run()
    nx, nb = 4 * 32, 2 * 64
    xbc = torch.full((c.T, nx + 2 * nb + 8), 3.0, device="cuda")
    xbc[:, :nx], xbc[:, nx:nx + nb], xbc[:, nx + nb:nx + 2 * nb] = \
        (dev(a.reshape(c.T, -1)) for a in (c.x, c.B, c.C))
    zd = torch.full((c.T, nx + 4), 3.0, device="cuda")
    zd[:, :nx], zd[:, nx:] = dev(c.z.reshape(c.T, -1)), dev(c.dt)
    st, wide = dev(c.state), torch.full((c.T, nx + 40), 7.0, device="cuda")
    w4.ssm_scan(w4.SeqPlan(i32(c.cu), c.n_slots, src=i32(c.src), dst=i32(c.dst)), xbc[:, :nx].unflatten(1, (4, 32)),
                zd[:, nx:], dev(c.A), xbc[:, nx:nx + nb].unflatten(1, (2, 64)),
                xbc[:, nx + nb:nx + 2 * nb].unflatten(1, (2, 64)), st, D=dev(c.D), z=zd[:, :nx].unflatten(1, (4, 32)),
                dt_bias=dev(c.bias), out=wide[:, 16:16 + nx].unflatten(1, (4, 32)))
    assert np.array_equal(wide[:, 16:16 + nx].cpu().numpy(), want[0].reshape(c.T, nx))
    assert np.array_equal(st.cpu().numpy(), want[1])
    assert bool((wide[:, :16] == 7).all()) and bool((wide[:, 16 + nx:] == 7).all())


def whole_numbers(c, keep=0.0):
    """Inputs that make every sum a small whole number: no decay, steps of 1,
    codes of -2 .. 2."""
    for k in ("x", "B", "C", "state"):
        v = getattr(c, k)
        v[...] = c.g.integers(-2, 3, v.shape)
    c.dt[...], c.A[...] = 1.0, keep
    c.softplus, c.bias, c.z = False, None, None
    if c.D is not None:
        c.D[...] = c.g.integers(-2, 3, c.D.shape)
    return c


@pytest.mark.parametrize("lens", [[5], [64], [65, 1, 200, 9], [640]])
@pytest.mark.parametrize("N,P,NH,NG", [(64, 64, 3, 1), (128, 64, 4, 2), (256, 16, 2, 2), (64, 48, 2, 1),
                                       (128, 128, 2, 1), (128, 16, 40, 8)])
def test_whole_numbers_are_exact(lens, N, P, NH, NG):
    whole_numbers(Case([13, N, P, *lens], lens, N=N, P=P, NH=NH, NG=NG)).check(exact=True)


@pytest.mark.parametrize("P,NH,lens", [(64, 128, [65, 9]), (80, 130, [70]), (32, 256, [20, 64]), (64, 128, [129])])
def test_enough_heads_for_wider_slices(P, NH, lens):
    """Calls with 32 columns for every compute unit: twice as many a workgroup;
    columns that end inside them."""
    whole_numbers(Case([26, P, *lens], lens, N=128, P=P, NH=NH, NG=2)).check(exact=True)
    Case([27, P, *lens], lens, N=128, P=P, NH=NH, NG=2, n_slots=len(lens), src=range(len(lens)),
         dst=range(len(lens))).check()


@pytest.mark.parametrize("n", [6, 200])
def test_strong_decay_forgets(n):
    """exp(-200) is 0 in fp32: a row's state is its own term."""
    whole_numbers(Case([14, n], [n]), keep=-200.0).check(exact=True)


@pytest.mark.parametrize("n", [8, 300])
def test_strong_and_weak_decays_in_turn(n):
    """Exponents of hundreds beside exponents near 0: the weak ones keep their
    precision though they are differences of long sums."""
    c = Case([15, n], [n], softplus=False, bias=False, N=128)
    c.A[...] = -1.0
    c.dt[...] = np.where(c.g.random(c.dt.shape) < 0.3, c.g.uniform(50, 300, c.dt.shape),
                         c.g.uniform(1e-4, 1e-2, c.dt.shape))
    c.check()


@pytest.mark.parametrize("n", [8, 150])
def test_steps_as_large_as_fp32_holds(n):
    """Decays whose exponents pass fp32's range are 0, and their sums no NaN."""
    c = Case([28, n], [n], softplus=False, bias=False, gate=False, D=False)
    c.dt[...] = np.where(c.g.random(c.dt.shape) < 0.3, np.float32(2e38), np.float32(1e-2))
    c.x *= np.float32(1e-3)
    c.check()


def test_no_decay_and_zero_steps():
    c = Case([16], [150, 5], softplus=False, bias=False)
    c.A[0] = 0.0
    c.dt[20:90] = 0.0
    c.dt[151] = 0.0
    c.check()


def test_growing_states():
    """A above 0: the state grows, within fp32's range."""
    c = Case([17], [150, 5], softplus=False, bias=False)
    c.A[...] = 0.5
    c.check()


def test_large_steps_of_softplus():
    """Softplus on both of its sides: very small steps, and steps as large as
    their argument."""
    c = Case([18], [70, 5])
    c.bias[...] = 0.0
    c.dt[...] = c.g.uniform(-40, 40, c.dt.shape)
    c.check()


def test_pieces_are_the_whole():
    c = Case([19], [300], N=128, n_slots=1, src=[-1], dst=[0])
    st, got, at = torch.full((1, 2, 128, 64), 5.0, device="cuda"), [], 0
    for i, n in enumerate((1, 60, 3, 130, 8, 98)):
        s = slice(at, at + n)
        plan = w4.SeqPlan(i32([0, n]), 1, src=i32([-1 if i == 0 else 0]), dst=i32([0]))
        got.append(w4.ssm_scan(plan, dev(c.x[s]), dev(c.dt[s]), dev(c.A), dev(c.B[s]), dev(c.C[s]), st, D=dev(c.D),
                               z=dev(c.z[s]), dt_bias=dev(c.bias)))
        at += n
    y = torch.cat(got).cpu().numpy()
    want, by, new, bs = ref.scan(c.cu, c.src, c.dst, c.x, c.dt, c.A, c.B, c.C, c.state, c.D, c.z, c.bias)
    assert np.all(np.abs(y - want) <= by) and np.all(np.abs(st.cpu().numpy() - new) <= bs)


def test_values_that_are_not_finite_stay_in_their_sequence_and_head():
    c = Case([20], [100, 100, 4], NH=3, NG=3, N=64, gate=False, n_slots=3, src=[-1] * 3, dst=[0, 1, 2])
    clean, cst = c.run()
    c.x[40, 1, 5], c.B[130, 2, 7], c.dt[202, 0] = np.nan, np.inf, np.nan
    y, st = c.run()
    hit = np.zeros(clean.shape, bool)
    hit[:100, 1], hit[100:200, 2], hit[200:, 0] = True, True, True
    assert np.array_equal(y[~hit], clean[~hit])
    assert np.isnan(y[40:100, 1, 5]).all() and np.isnan(y[202:, 0]).all()
    sh = np.zeros(cst.shape, bool)
    sh[0, 1], sh[1, 2], sh[2, 0] = True, True, True
    assert np.array_equal(st[~sh], cst[~sh])


def test_state_that_is_not_finite_stays_in_its_sequence():
    c = Case([21], [70, 70, 2, 2])
    clean, cst = c.run()
    c.state[c.src[0], 1, 3, 9] = np.nan
    c.state[c.src[2], 0, 3, 9] = np.inf
    y, st = c.run()
    a, b = slice(0, 70), slice(140, 142)
    rest = np.ones(len(y), bool)
    rest[a], rest[b] = False, False
    assert np.array_equal(y[rest], clean[rest])
    assert not np.isfinite(y[a, 1, 9]).any() and not np.isfinite(y[b, 0, 9]).any()


@pytest.mark.parametrize("lens", [[1] * 5, [300, 7], [64] * 6])
def test_equal_bits_from_call_to_call(lens):
    c = Case([22, *lens], lens, NH=8, N=128)
    want = c.run()
    ws = torch.randint(0, 255, (1 << 22,), dtype=torch.uint8, device="cuda")     # any contents
    for _ in range(3):
        got = c.run(workspace=ws)
        assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_many_sequences():
    g = np.random.default_rng(23)
    Case([23], list(g.integers(0, 3, 700)), NH=1, P=16).check()
    Case([24], list(g.integers(0, 30, 100)), NH=1, P=16).check()


def test_long_sequence():
    Case([25], [2500, 5], NH=1, P=32, N=128).check()


# (up to 1024 sequences are taken longest first, more as they come)
@pytest.mark.parametrize("B", [3, 64, 255, 257, 1024, 1025, 1300])
def test_long_sequences_anywhere_among_short_ones(B):
    g = np.random.default_rng([30, B])
    lens = g.choice([0, 1, 3, 9, 64, 70, 193], B, p=[0.2, 0.4, 0.2, 0.08, 0.04, 0.04, 0.04])
    lens[-1] = 260
    Case([31, B], lens, NH=1, P=16).check()


@pytest.mark.parametrize("order", [1, -1])
def test_long_sequences_in_either_order_with_wide_slices(order):
    lens = [330, 200, 200, 129, 64, 9, 1, 0][::order]
    Case([32], lens, NH=40, P=64, N=128).check()
