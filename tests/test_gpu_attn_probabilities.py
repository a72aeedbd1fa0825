"""stree_tree_attn in bf16 with up to 16 rows to a key/value head: probabilities count with 15 bits, not with bf16's 8."""
import numpy as np
import pytest

from kv_helpers import HALF, attn_bound, within
from test_gpu_tree_attn import _case, _run, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H,G,P,lens", [(1, 4, 1, 64, [31, 300]), (1, 8, 2, 128, [2000, 5, 64]), (4, 4, 1, 128, [33, 500]), (1, 16, 1, 80, [100, 700]),
                                          (2, 6, 1, 256, [90, 1000]), (16, 1, 1, 64, [40, 257])])
def test_probabilities_between_two_bf16_values(N, H, G, P, lens):
    """Keys of weight 1 with values of -1, two of three with a weight just short of the middle between two bf16 values and values of
    1: what is left of the sums is what the weights' lower bits make of it."""
    c = _case(P + N, "bf16", N, H, G, P, 16, lens)
    p = 0.5 + 0.98 * 2.0 ** -9                              # (its neighbours are 0.5 and 0.5 + 2^-8)
    c["q"] = np.zeros_like(c["q"])
    c["q"][..., 0] = 1
    k, v = c["k"], c["v"]
    k[~np.isnan(k)], v[~np.isnan(v)] = 0, -1
    for b, n in enumerate(lens):
        t = np.arange(n + N)
        t = t[t % 3 > 0]
        pg = c["table"][b, t // 16]
        k[pg, :, t % 16, 0] = -1
        v[pg, :, :, t % 16] = 1
    scale = -float(np.log(p))
    want, status, weight, score = _want(c, scale)
    got, gs = _run(c, scale=scale)
    assert not status.any() and not gs.any()
    # one rounding of the result; 15 bits of a probability above and below the fraction line: a part p (1 - 2^-8), rounded by up to
    # 2^-8 of it, leaves up to 2 2^-8 p, which is rounded by up to 2^-8 of that; fp32 sums of P and of all products
    bits = 2 * HALF["bf16"] ** 2
    s = (P + 8) * HALF["f32"] * score[..., None] + 8 * HALF["f32"]
    bound = HALF["bf16"] * np.abs(want) * (1 + 2 * bits) + 2 * (bits + s + (max(lens) + N) * HALF["f32"]) * weight
    assert (bound < 1e-3).all()
    within(got, want, bound, "attention")


@pytest.mark.parametrize("io,N,R,P", [("bf16", 1, 4, 128), ("bf16", 3, 4, 80), ("bf16", 16, 1, 64), ("bf16", 2, 4, 256), ("bf16", 6, 4, 128), ("bf16", 20, 4, 64),
                                      ("bf16", 80, 4, 128), ("f32", 1, 4, 128), ("f32", 8, 4, 40)])
def test_infinite_values_of_the_text_stay_infinite(io, N, R, P):
    """All weights are above zero: a column with one infinite value is infinite, one with both is NaN, whatever a weight's lower bits
    are (those of the largest, 1, are zeros)."""
    c = _case(N * 3 + P, io, N, R, 1, P, 16, [150, 7])
    for b, t, col, value in ((0, 5, 0, np.inf), (0, 140, 3, -np.inf), (0, 33, P - 1, np.inf), (0, 90, P - 1, -np.inf), (1, 2, 1, np.inf), (1, 6, 1, np.inf)):
        c["v"][c["table"][b, t // 16], 0, col, t % 16] = value
    with np.errstate(invalid="ignore"):
        want, status, weight, score = _want(c)
    assert not status.any() and np.isposinf(want[0, ..., 0]).all() and np.isneginf(want[0, ..., 3]).all() and np.isnan(want[0, ..., P - 1]).all()
    assert np.isposinf(want[1, ..., 1]).all() and np.isfinite(want[1, ..., 0]).all()
    inside = np.isfinite(want)
    bound = attn_bound(io, np.where(inside, want, 0), np.where(inside, weight, 0), score, P, 150 + N)
    for plain in (True, False):
        got, gs = _run(c, plain=plain)
        assert not gs.any()
        assert np.array_equal(got[~inside], want[~inside].astype(np.float32), equal_nan=True), plain
        within(np.where(inside, got, 0), np.where(inside, want, 0), bound, f"plain {plain}")
