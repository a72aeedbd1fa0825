"""stree_tree_attn where its work is cut differently: numbers of rows around the tile sizes, batches beyond a wave, rows that see
less of a piece than others, empty calls; infinities and NaN on every kernel."""
import numpy as np
import pytest

from kv_helpers import attn_bound, dev, within
from oracle import paged
from paper_2505_14969_amd import binding as st
from test_gpu_tree_attn import _case, _check, _run, _want

pytestmark = pytest.mark.gpu


# rows of a key/value head: nodes x queries a head; 16 and 32 of the streaming kernel, 64 and 256 of the one that shares tiles
@pytest.mark.parametrize("P,page", [(64, 16), (128, 16), (128, 64), (64, 256), (96, 32)])
@pytest.mark.parametrize("N,R", [(1, 15), (1, 17), (2, 16), (11, 3), (8, 5), (16, 4), (13, 5), (32, 4), (43, 3), (64, 4), (257, 1), (128, 3), (100, 6)])
def test_rows_around_the_tiles(N, R, P, page):
    _check(_case(N * R, "bf16", N, R, 1, P, page, [130, 0, 700], tree="random" if N <= 256 else "chain"), plain=(False,))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,N", [(64, 1), (65, 1), (300, 1), (257, 3), (700, 2)])
def test_batches(io, B, N):
    """More sequences than lanes of a wave, and than threads of a workgroup: idle ones, bad ones and lengths of all sizes."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 90, B)
    lens[rng.random(B) < 0.1] = -1
    lens[::50] = 900
    c = _case(B, io, N, 4, 2, 64, 16, list(lens))
    for b in (3, B - 1):
        c["table"][b, 0] = 1 << 20
    if N > 1:
        c["parent"][5, 1] = 1
    _check(c, plain=(False,))


def test_batch_of_long_and_short():
    _check(_case(5, "bf16", 1, 8, 2, 128, 16, [6000] + [5] * 80 + [3000]), plain=(False,))


@pytest.mark.parametrize("N,R,P", [(4, 4, 128), (10, 3, 64), (20, 3, 128), (40, 2, 64), (90, 4, 128)])
def test_infinities_and_nan_on_every_kernel(N, R, P):
    """Nodes whose keys or values are not finite spoil the rows that see them and no others, whatever the tile."""
    for io in ("bf16", "f32"):
        c = _case(N, io, N, R, 1, P, 16, [45, 100])
        for i, (node, what, value) in enumerate(((1, "v", np.nan), (N - 1, "k", np.nan), (N // 2, "v", -np.inf), (N - 2, "v", np.inf))):
            t = 45 + node
            pg = c["table"][0, t // 16]
            (c["k"][pg, 0, t % 16] if what == "k" else c["v"][pg, 0, :, t % 16])[2 + i] = value
        got, status = _run(c)
        with np.errstate(invalid="ignore"):
            want, ws, weight, score = _want(c)
        assert np.array_equal(status, ws)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
        inside = np.isfinite(want)
        assert np.array_equal(got[~inside & ~np.isnan(want)], want[~inside & ~np.isnan(want)])
        bound = attn_bound(io, want, weight, np.where(np.isfinite(score), score, 0), P, 200)
        assert np.all(np.abs(got[inside] - want[inside]) <= bound[inside]) and not inside[0].all() and inside[1].all()


@pytest.mark.parametrize("io,N,R", [("bf16", 700, 1), ("f32", 100, 1), ("bf16", 40, 1)])
def test_a_bad_page_that_only_late_rows_see(io, N, R):
    """The last page's number is bad: zeros for all rows of the sequence, the first ones' too, whose keys end before it."""
    c = _case(N, io, N, R, 1, 64, 16, [0, 20], tree="chain")
    c["table"][0, (N - 1) // 16] = -7
    got, status = _run(c)
    assert list(status) == [st.SEQ_PAGE, 0] and not got[0].any() and np.isfinite(got[1]).all() and got[1].any()
    want, _, weight, score = _want(c)
    within(got, want, attn_bound(io, want, weight, score, 64, N + 20), "the other sequence")


@pytest.mark.parametrize("io,N,R", [("bf16", 1, 4), ("bf16", 30, 1), ("bf16", 20, 4), ("bf16", 64, 4), ("f32", 20, 4)])
def test_large_scores(io, N, R):
    """One key that takes all, first seen early or late: the running maximum moves by far."""
    c = _case(N, io, N, R, 1, 128, 16, [400, 33])
    c["q"] = c["q"] * 8
    for b, t in ((0, 350), (1, 2)):
        pg = c["table"][b, t // 16]
        c["k"][pg, 0, t % 16] = np.sign(c["q"][b, 0, 0]) * 8
    _check(c, plain=(False,))


def test_empty_batch():
    import torch
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    k, v, q = z(3, 2, 16, 64), z(3, 2, 64, 16), z(0, 5, 4, 64)
    assert st.stree_tree_attn(i(0, 5), i(0), q, k, v, i(0, 4)).shape == q.shape
    kv = z(0, 5, 2, 64)
    assert st.stree_tree_rope(None, i(0), q, kv, kv, k, v, i(0, 4), torch.zeros(32, dtype=torch.float64, device="cuda")).shape == q.shape
    assert st.stree_commit_kv(i(0, 5), i(0), i(0), k, v, i(0, 4)).shape == (0,)
    st.stree_resize_kv(i(0), i(0), i(0, 4), i(3), i(3), i(1), 16)
    assert st.stree_fork_kv(i(0), i(0), i(2), i(2), i(2, 4), i(3), i(3), i(1), k, v).shape == (0,)
    torch.cuda.synchronize()


def test_one_page_of_text_and_a_table_of_one_entry():
    """A table that reaches one page: no parts, no scratch."""
    c = _case(3, "bf16", 6, 4, 2, 64, 128, [100, 122, 0])
    o = lambda a: dev("bf16", a)  # noqa: E731
    assert st.stree_attn_workspace(o(c["q"]), o(c["k"]), o(c["v"]), o(c["table"])) == 0
    _check(c)
    assert paged.LENGTH == st.SEQ_LENGTH and paged.PAGE == st.SEQ_PAGE and paged.HELD == st.SEQ_HELD
