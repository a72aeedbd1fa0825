"""stree_tree_attn: a bad page number that lies far behind the last key of a tile's rows, in a head that a workgroup comes to after
another one: the whole sequence gets zeros and its status, whichever kernel takes it."""
import numpy as np
import pytest

from kv_helpers import attn_bound, within
from paper_2505_14969_amd import binding as st
from test_gpu_tree_attn import _case, _run, _want

pytestmark = pytest.mark.gpu


# The rows make more tiles than the chip holds workgroups, so that each goes through every head of both sequences, the second
# sequence's first head behind a tile that saw all keys of the one before.  Entry 100 is more than 64 behind a first tile's keys.
@pytest.mark.parametrize("io,N,H,G,P,entry", [("f32", 2100, 8, 2, 64, 100), ("bf16", 2100, 8, 2, 80, 100), ("bf16", 4200, 4, 2, 32, 200),
                                              ("f32", 1300, 16, 2, 24, 70), ("bf16", 2100, 8, 2, 64, 100)])
def test_a_bad_page_far_behind_the_first_rows(io, N, H, G, P, entry):
    c = _case(N + P, io, N, H, G, P, 16, [0, 0], tree="chain")
    c["table"][1, entry] = -7
    got, status = _run(c)
    assert list(status) == [0, st.SEQ_PAGE]
    assert not got[1].any(), "zeros for all of the sequence's rows"
    # the other sequence: its first rows and its last ones
    c = {**c, "lens": c["lens"][:1], "table": c["table"][:1], "q": c["q"][:1]}
    some = np.r_[0:4, N - 3:N]
    for i in some:
        part = {**c, "lens": np.array([i], np.int32), "q": c["q"][:, i:i + 1], "parent": None}
        want, _, weight, score = _want(part)
        within(got[:1, i:i + 1], want, attn_bound(io, want, weight, score, P, N), f"node {i}")
