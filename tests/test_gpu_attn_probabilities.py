"""stree_tree_attn in bf16 with up to 16 rows to a key/value head: probabilities count with 16 bits, not with bf16's 8."""
import numpy as np
import pytest

from kv_helpers import HALF, within
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
    # one rounding of the result; 16 bits of a probability above and below the fraction line; fp32 sums of P and of all products
    bits = HALF["bf16"] ** 2
    s = (P + 8) * HALF["f32"] * score[..., None] + 8 * HALF["f32"]
    bound = HALF["bf16"] * np.abs(want) * (1 + 2 * bits) + 2 * (bits + s + (max(lens) + N) * HALF["f32"]) * weight
    assert (bound < 1e-3).all()
    within(got, want, bound, "attention")
