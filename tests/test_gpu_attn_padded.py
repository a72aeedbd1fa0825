"""stree_tree_attn with heads that are no whole 64, 128 or 256 columns: keys with infinities in any of their columns."""
import numpy as np
import pytest

from kv_helpers import attn_bound, within
from test_gpu_tree_attn import _case, _run, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io,N,P", [("bf16", 1, 80), ("bf16", 12, 80), ("bf16", 3, 96), ("bf16", 9, 40), ("bf16", 2, 200), ("bf16", 5, 8), ("bf16", 20, 128),
                                    ("f32", 1, 96), ("f32", 12, 20), ("f32", 4, 136), ("f32", 9, 4), ("f32", 5, 60)])
def test_infinite_keys_weigh_nothing_or_everything(io, N, P):
    """A score of -inf leaves the row as if the key were not there, one of +inf makes it NaN, as the formula does: heads 0 and 1 have
    one sign in every column, heads 2 and 3 the other.  Columns at the front, in the middle and at the end; text and nodes."""
    c = _case(N * 131 + P, io, N, 4, 1, P, 16, [70, 200, 33, 130, 5])
    sign = np.array([1, 1, -1, -1], np.float32)
    c["q"] = (np.abs(c["q"]) + np.float32(0.5)) * sign[:, None]
    put = [(0, 5, 0, -np.inf), (1, 150, min(7, P - 1), np.inf), (2, 32, P - 1, -np.inf), (3, 0, P // 2, np.inf), (4, 5, 1, -np.inf)]     # (the last: a root)
    clean = {**c, "k": c["k"].copy()}
    for b, t, col, value in put:
        pg = c["table"][b, t // 16]
        c["k"][pg, 0, t % 16, col] = value
        clean["k"][pg, 0, t % 16, col] = 0
    with np.errstate(invalid="ignore"):
        want, status, weight, _ = _want(c)
    score = _want(clean)[3]                                 # (rounding errors of the finite scores; the others have none)
    assert not status.any()
    # sequences 0, 2 and 4: -inf for heads 0 and 1; 1 and 3: for heads 2 and 3
    for b in range(5):
        alive = slice(0, 2) if b % 2 == 0 else slice(2, 4)
        dead = slice(2, 4) if b % 2 == 0 else slice(0, 2)
        assert np.isfinite(want[b, 1:, alive]).all() and np.isnan(want[b, :, dead]).all()
    bound = attn_bound(io, want, weight, score, P, 200 + N)
    for plain in (True, False):
        got, gs = _run(c, plain=plain)
        assert not gs.any()
        within(got, want, bound, f"plain {plain}")
