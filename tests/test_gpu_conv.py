"""The short causal convolution against the plain form in 64 bits (GPU)."""
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
    """Random inputs for sequences of these lengths, after `lead` rows of
    none and before `tail` such rows."""

    def __init__(self, seed, lens, CH, W, bias=True, lead=0, tail=0, n_slots=None, src=None, dst=None):
        g = self.g = np.random.default_rng(seed)
        self.cu = lead + np.concatenate([[0], np.cumsum(lens)])
        self.T = int(self.cu[-1]) + tail
        self.n_slots = 2 * len(lens) if n_slots is None else n_slots
        slots = g.permutation(max(self.n_slots, 2 * len(lens)))
        self.src = slots[:len(lens)] if src is None else np.asarray(src)
        self.dst = slots[len(lens):2 * len(lens)] if dst is None else np.asarray(dst)
        self.x = g.standard_normal((self.T, CH)).astype(np.float32)
        self.w = g.standard_normal((W, CH)).astype(np.float32)
        self.bias = g.standard_normal(CH).astype(np.float32) if bias else None
        self.state = g.standard_normal((self.n_slots, W - 1, CH)).astype(np.float32)

    def run(self, act="silu", x=None, out=None, rows=None, **kw):
        plan = w4.SeqPlan(i32(self.cu), self.n_slots, src=i32(self.src), dst=i32(self.dst))
        st = dev(self.state)
        T = self.T if rows is None else rows
        if out is None:
            out = torch.full((T, self.x.shape[1]), 7.0, device="cuda")
        x = dev(self.x)[:T] if x is None else x
        w4.short_conv(plan, x, dev(self.w), st if self.n_slots else None, bias=dev(self.bias), act=act, out=out, **kw)
        return out.cpu().numpy(), st.cpu().numpy()

    def check(self, act="silu", rows=None, **kw):
        y, st = self.run(act, rows=rows, **kw)
        T = self.T if rows is None else rows
        want, bound, new = ref.conv(self.cu, self.src, self.dst, self.x[:T], self.w, self.bias, self.state, act)
        none = np.isnan(want)
        assert np.all(y[none] == 7.0), "rows of no sequence"
        err = np.abs(y - want)
        assert np.all(err[~none] <= bound[~none]), np.argwhere(~none & ~(err <= bound))[:5]
        assert np.array_equal(st, new), np.argwhere(st != new)[:5]


# one row to several runs of rows; sequences that begin and end anywhere in
# a run, shorter than the history, empty
@pytest.mark.parametrize("lens", [[1], [2], [3], [4], [16], [17], [100], [1, 1, 1, 1, 1], [14, 3, 1, 2, 40, 1],
                                  [0, 5, 0, 0, 33, 0], [15, 1, 15, 2, 16, 3], [63, 64, 65, 1], [700]])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_lengths(lens, W):
    Case([1, W, *lens], lens, 72, W).check()


@pytest.mark.parametrize("CH", [4, 60, 256, 260, 1028, 4352])
@pytest.mark.parametrize("act,bias", [("silu", False), ("none", True)])
def test_channels(CH, act, bias):
    Case([2, CH], [9, 1, 30], CH, 4, bias=bias).check(act)


@pytest.mark.parametrize("W", [2, 4])
def test_rows_of_no_sequence_are_left(W):
    Case([3, W], [5, 0, 21], 64, W, lead=6, tail=19).check()


@pytest.mark.parametrize("rows", [1, 2, 3, 17, 20, 35])
def test_calls_with_fewer_rows_than_the_plan(rows):
    """The call has the first rows; states are those after them."""
    Case([4, rows], [18, 1, 20], 64, 4).check(rows=rows)


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("n", [1, 2, 16, 17, 50])
def test_state_in_place(W, n):
    Case([5, W, n], [n, n + 1, 2], 520, W, n_slots=3, src=[2, 0, 1], dst=[2, 0, 1]).check()


def test_absent_slots_begin_with_zeros_and_keep_nothing():
    Case([6], [7, 8, 9, 2], 64, 4, n_slots=4, src=[-1, 1, 4, 2], dst=[0, -1, 3, 1 << 30]).check()


def test_default_slots():
    c = Case([7], [7, 2, 9], 64, 4, n_slots=3, src=[0, 1, 2], dst=[0, 1, 2])
    want = c.run()
    plan = w4.SeqPlan(i32(c.cu), 3)
    st = dev(c.state)
    y = w4.short_conv(plan, dev(c.x), dev(c.w), st, bias=dev(c.bias))
    assert np.array_equal(y.cpu().numpy(), want[0]) and np.array_equal(st.cpu().numpy(), want[1])
    # dst by default the slot read
    c.src, c.dst = np.array([2, 0, 1]), np.array([2, 0, 1])
    want = c.run()
    st = dev(c.state)
    y = w4.short_conv(w4.SeqPlan(i32(c.cu), 3, src=i32(c.src)), dev(c.x), dev(c.w), st, bias=dev(c.bias))
    assert np.array_equal(y.cpu().numpy(), want[0]) and np.array_equal(st.cpu().numpy(), want[1])


def test_no_slots_at_all():
    c = Case([8], [7, 20], 64, 4, n_slots=0, src=[0, -1], dst=[0, 1])
    c.state = np.zeros((0, 3, 64), np.float32)
    c.check()


def test_several_sequences_read_one_slot():
    Case([9], [7, 20, 3], 64, 4, n_slots=5, src=[1, 1, 1], dst=[0, 2, 4]).check()


def test_strided_rows():
    c = Case([10], [7, 20, 3], 64, 4)
    wide = torch.full((c.T, 164), 3.0, device="cuda")
    wide[:, 20:84] = dev(c.x)
    o = torch.full((c.T, 100), 7.0, device="cuda")
    c.check(x=wide[:, 20:84], out=o[:, 16:80])
    assert bool((o[:, :16] == 7).all()) and bool((o[:, 80:] == 7).all())


def test_pieces_are_the_whole():
    """One sequence in pieces of any length through its state: equal bits."""
    c = Case([11], [60], 64, 4, n_slots=1, src=[-1], dst=[0])
    whole, last = c.run()
    st = torch.zeros(1, 3, 64, device="cuda")
    got, at = [], 0
    for i, n in enumerate((1, 1, 2, 1, 5, 17, 3, 30)):
        plan = w4.SeqPlan(i32([0, n]), 1, src=i32([-1 if i == 0 else 0]), dst=i32([0]))
        got.append(w4.short_conv(plan, dev(c.x[at:at + n]), dev(c.w), st, bias=dev(c.bias)))
        at += n
    assert np.array_equal(torch.cat(got).cpu().numpy(), whole) and np.array_equal(st.cpu().numpy(), last)


def test_values_that_are_not_finite_reach_their_own_rows_only():
    c = Case([12], [12, 12], 64, 4, n_slots=2, src=[-1, -1], dst=[0, 1])
    clean, _ = c.run("none")
    c.x[5, 3], c.x[11, 7] = np.nan, np.inf
    y, st = c.run("none")
    hit = np.zeros_like(clean, bool)
    hit[5:9, 3], hit[11, 7] = True, True
    assert np.array_equal(y[~hit], clean[~hit]) and not np.isfinite(y[hit]).any()
    assert np.isinf(st[0, 2, 7]) and np.isfinite(st[1]).all()


def test_large_arguments_of_silu():
    c = Case([13], [12], 64, 4)
    c.x *= 60.0
    c.check()


def test_many_sequences():
    g = np.random.default_rng(14)
    Case([14], list(g.integers(0, 4, 3000)), 64, 4).check()
