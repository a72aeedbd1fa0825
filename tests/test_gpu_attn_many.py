"""stree_tree_attn: many sequences of many rows each, where a workgroup's share goes over several of them; single rows of odd strides."""
import numpy as np
import pytest

from kv_helpers import attn_bound, dev, within
from paper_2505_14969_amd import binding as st
from test_gpu_tree_attn import _case, _check, _run, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,N,R,P,page", [(66, 20, 4, 64, 16), (300, 9, 4, 128, 32), (70, 70, 4, 64, 64), (520, 33, 1, 64, 16), (130, 65, 2, 128, 128)])
def test_many_sequences_of_many_rows(B, N, R, P, page):
    """Idle ones, bad trees and bad pages among lengths of all sizes; trees of up to 64 nodes and of more."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 200, B)
    lens[rng.random(B) < 0.1] = -1
    lens[::50] = 700
    lens[[3, 5, B - 1]] = (40, 130, 1)
    c = _case(B, "bf16", N, R, 1, P, page, list(lens))
    c["table"][3, 0] = -2
    c["table"][B - 1, (int(lens[B - 1]) + N - 1) // page] = 1 << 30
    c["parent"][5, N - 1] = N - 1
    _check(c, plain=(False,))


@pytest.mark.parametrize("io,N,R,lens", [("bf16", 2100, 4, [1, 0]), ("bf16", 1100, 4, [70, -1, 3]), ("bf16", 800, 3, [0, 900]), ("f32", 700, 4, [5, 0]),
                                         ("f32", 300, 4, [1000]), ("bf16", 130, 1, [64, 63, 65])])
def test_long_prompts(io, N, R, lens):
    """Tiles of rows that see ever more keys, more of them than leave a worker for every eighth of the chip."""
    _check(_case(N, io, N, 2 * R, 2, 64, 64, lens, tree="chain"), plain=(False,))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_infinities_in_a_prompt(io):
    """A prompt's token whose values are not finite: the rows in front of it do not see them, all others do, whatever tile they are in."""
    c = _case(6, io, 400, 4, 1, 64, 16, [37, 20], tree="chain")
    for node, value, col in ((100, np.inf, 3), (250, -np.inf, 3), (131, np.nan, 60), (399, np.inf, 9)):
        t = 37 + node
        c["v"][c["table"][0, t // 16], 0, col, t % 16] = value
    got, status = _run(c)
    assert not status.any()
    with np.errstate(invalid="ignore"):
        want, _, weight, score = _want(c)
    for col, first in ((60, 131), (9, 399)):
        assert np.isfinite(got[0, :first, :, col]).all() and not np.isfinite(got[0, first:, :, col]).any()
    assert np.isfinite(got[0, :100, :, 3]).all() and (got[0, 100:250, :, 3] == np.inf).all() and np.isnan(got[0, 250:, :, 3]).all()
    inside = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), inside)
    bound = attn_bound(io, want, weight, score, 64, 437)
    assert np.all(np.abs(got[inside] - want[inside]) <= bound[inside])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_one_row_of_any_stride(io):
    """One node of one sequence: its row's distance to a next one, which is not there, means nothing."""
    c = _case(1, io, 1, 4, 2, 64, 16, [77])
    args = [dev(io, c[x]) for x in ("lens", "q", "k", "v", "table")]
    want = st.stree_tree_attn(None, *args)
    for q in (args[1].as_strided(args[1].shape, (0, 0, 64, 1)), args[1].as_strided(args[1].shape, (7, 3, 64, 1))):
        assert np.array_equal(st.stree_tree_attn(None, args[0], q, *args[2:]).float().cpu().numpy(), want.float().cpu().numpy())
    exact, _, weight, score = _want(c)
    within(want.double().cpu().numpy(), exact, attn_bound(io, exact, weight, score, 64, 78), "the row")
