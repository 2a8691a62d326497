"""The state space scan on plans with places to spare (more sequences than rows,
most of them empty): long sequences go by chunks all the same, which shows in what
the call writes to its workspace (GPU)."""
import functools

import numpy as np
import pytest

import paper_2606_24031_amd as w4

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from tests.test_gpu_ssm import Case, i32


def check(c, N, P, NH):
    """Within the bounds; returns whether the workspace was written."""
    plan = w4.SeqPlan(i32(c.cu), c.n_slots)
    ws = torch.full((w4.ssm_workspace(plan, c.T, NH, 1, N, P).numel(),), 171, dtype=torch.uint8, device="cuda")
    c.run = functools.partial(c.run, workspace=ws)
    c.check()
    return not bool((ws == 171).all())


@pytest.mark.parametrize("at", [0, 500, 1023])
@pytest.mark.parametrize("N,P", [(64, 32), (128, 64), (256, 16)])
def test_one_prompt_in_a_large_plan(at, N, P):
    lens = [0] * 1024
    lens[at] = 947
    assert check(Case([50, at, N], lens, NH=1, N=N, P=P), N, P, 1)


@pytest.mark.parametrize("B", [300, 1024, 1025, 1500])
def test_prompts_and_tokens_in_a_large_plan(B):
    """Up to 1024 sequences are taken longest first, more as they come."""
    lens = np.zeros(B, int)
    lens[[5, 17, 18, B - 1]] = 129, 65, 8, 9
    lens[20:60] = 1
    lens[100:104] = 2
    assert check(Case([51, B], list(lens), NH=2, P=16), 64, 16, 2)


def test_as_many_sequences_as_rows():
    """Taken to be single tokens, in one launch: right for any others too."""
    for lens in ([70] + [0] * 69, [1] * 60 + [40] + [0] * 39, [0, 1] + [1] * 97 + [2]):
        assert not check(Case([52, *lens], lens, NH=2, P=32, N=128), 128, 32, 2)


@pytest.mark.parametrize("n", [31, 32, 33, 34])
def test_about_the_bound(n):
    lens = [0] * 100
    lens[2], lens[50], lens[98] = n, 66 - n, 3
    check(Case([55, n], lens, NH=2, P=32, N=128), 128, 32, 2)


def test_rows_up_to_a_chunk_stay_one_launch():
    for lens in ([64] + [0] * 80, [0] * 30 + [20], [1] * 64 + [0] * 9):
        assert not check(Case([53, *lens], lens, NH=2, P=32, N=128), 128, 32, 2)


def test_calls_with_fewer_rows_than_a_large_plan():
    lens = [0] * 200
    lens[3], lens[100], lens[150] = 100, 50, 50
    Case([54], lens, NH=2, P=16).check(rows=130)


def test_a_graph_whose_plan_changes_between_replays():
    """Captured once with places to spare, replayed with a prompt, with tokens, with
    both, with neither: each replay as the same call made eagerly."""
    B, T = 130, 100
    plans = [[100], [1] * 100, [3, 40, 1, 33, 2, 21], [0] * 130, [32, 33, 35], [1] * 20 + [60]]
    c = Case([56], [100] + [0] * (B - 1), NH=2, P=32, N=128, n_slots=B, src=range(B), dst=range(B))
    dev = lambda a: torch.from_numpy(a).cuda()
    x, z, dt, A, b, cc = map(dev, (c.x, c.z, c.dt, c.A, c.B, c.C))
    cu, st, out = i32(np.zeros(B + 1)), dev(c.state), torch.zeros(T, 2, 32, device="cuda")
    plan = w4.SeqPlan(cu, B)
    ws = w4.ssm_workspace(plan, T, 2, 1, 128, 32)
    call = lambda: w4.ssm_scan(plan, x, dt, A, b, cc, st, z=z, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for lens in plans * 2:
        ends = np.concatenate([[0], np.cumsum(lens + [0] * (B - len(lens)))])
        got = []
        for f in (call, g.replay):
            cu.copy_(i32(ends))
            st.copy_(dev(c.state))
            out.fill_(7.0)
            f()
            torch.cuda.synchronize()
            got.append((out.clone(), st.clone()))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert bool((got[0][0][sum(lens):] == 7).all())
