"""stree_tree_rope against the fp64 form: norms, rotation, rows appended to the cache, and what is left as it was."""
import numpy as np
import pytest

from kv_helpers import HALF, caches, dev, host, rounded, tables, trees, within
from oracle import paged
from paper_2505_14969_amd import binding as st

pytestmark = pytest.mark.gpu


def _case(seed, io, B, N, H, G, P, page, lens, R, tree="random", interleaved=False, norms=True, scale=1.0, width=None):
    rng = np.random.default_rng(seed)
    lens = np.array(lens, np.int32)
    table, npages = tables(rng, lens, N, page, width=width)
    k_cache, v_cache = caches(rng, io, lens, 0, table, npages, G, P, page)
    rows = rounded(io, rng.standard_normal((B, N, (H + 2 * G) * P)) * 2)
    turns = 500000.0 ** (-np.arange(R // 2) / max(R // 2, 1)) / (2 * np.pi)
    qn = rounded(io, rng.uniform(0.5, 1.5, P)) if norms else None
    kn = rounded(io, rng.uniform(0.5, 1.5, P)) if norms else None
    return dict(io=io, parent=trees(rng, B, N, tree), lens=lens, rows=rows, k=k_cache, v=v_cache, table=table, turns=turns, qn=qn, kn=kn,
                inter=interleaved, scale=scale, H=H, G=G, P=P)


def _split(rows, H, G, P):
    cut = lambda a, b: rows[..., a * P:b * P].reshape(*rows.shape[:2], b - a, P) if isinstance(rows, np.ndarray) else rows[..., a * P:b * P].unflatten(2, (b - a, P))  # noqa: E731
    return cut(0, H), cut(H, H + G), cut(H + G, H + 2 * G)


def _run(c, out=None, eps=1e-6):
    import torch
    io = c["io"]
    o = lambda a: None if a is None else dev(io, a)  # noqa: E731
    q, k, v = _split(dev(io, c["rows"]), c["H"], c["G"], c["P"])
    kc, vc = dev(io, c["k"]), dev(io, c["v"])
    status = torch.full((len(c["lens"]),), 77, dtype=torch.int32, device="cuda")
    got = st.stree_tree_rope(o(c["parent"]), o(c["lens"]), q, k, v, kc, vc, o(c["table"]), o(c["turns"]), o(c["qn"]), o(c["kn"]), eps,
                             c["inter"], c["scale"], status=status)
    return host(got), host(kc), host(vc), host(status)


def _check(c, eps=1e-6):
    q, k, v = _split(c["rows"], c["H"], c["G"], c["P"])
    wk, wv = c["k"].astype(np.float64), c["v"].astype(np.float64)
    want, status, size_q, size_k = paged.rope(c["parent"], c["lens"], q, k, v, wk, wv, c["table"], c["turns"], c["qn"], c["kn"], eps,
                                              c["inter"], c["scale"])
    got, gk, gv, gs = _run(c, eps=eps)
    assert np.array_equal(gs, status)
    # rounding of the result, and of fp32: the norm (a sum of P squares, a root, two products), cosine and sine and
    # their products, relative to |u| + |w|
    fine = (c["P"] / 2 + 24) * HALF["f32"]
    within(got, want, HALF[c["io"]] * (1 + fine) * np.abs(want) + fine * size_q, "q")
    B, N = q.shape[:2]
    bound = np.zeros(wk.shape)
    page = wk.shape[2]
    for b in range(B):
        if status[b] == 0 and c["lens"][b] >= 0:
            t = np.arange(c["lens"][b], c["lens"][b] + N)
            pg = c["table"][b, t // page]
            bound[pg, :, t % page] = HALF[c["io"]] * (1 + fine) * np.abs(wk[pg, :, t % page]) + fine * size_k[b]
    within(gk, wk, bound, "keys")                          # (unwritten slots: as they were, NaN)
    assert np.array_equal(gv, wv.astype(np.float32), equal_nan=True), "values are copied"


CASES = [
    # io, B, N, H, G, P, page, lengths, rotary
    ("bf16", 1, 1, 32, 8, 128, 16, [1003], 128), ("bf16", 1, 1, 4, 4, 64, 16, [0], 64), ("f32", 1, 1, 8, 2, 128, 32, [15], 128),
    ("bf16", 3, 15, 32, 8, 128, 16, [0, 1, 47], 128), ("bf16", 2, 64, 8, 2, 128, 64, [63, 200], 64), ("bf16", 2, 256, 4, 1, 64, 16, [5, 16], 64),
    ("f32", 2, 100, 6, 3, 80, 128, [127, 128], 80), ("bf16", 4, 17, 5, 5, 96, 16, [31, -1, 33, 7], 32), ("f32", 1, 33, 3, 1, 20, 16, [9], 10),
    ("bf16", 2, 31, 7, 7, 40, 256, [250, 3], 8), ("bf16", 1, 65, 4, 2, 256, 16, [100], 256), ("f32", 2, 3, 2, 1, 33, 16, [14, 15], 32),
    ("bf16", 1, 9, 3, 1, 24, 16, [8], 24), ("bf16", 1, 5, 2, 1, 7, 16, [13], 6), ("f32", 3, 16, 4, 2, 128, 16, [16, 8, 24], 0),
    ("bf16", 2, 48, 64, 8, 128, 16, [90, 1], 128), ("f32", 1, 2, 2, 2, 4, 16, [15], 4), ("bf16", 1, 4, 2, 2, 1, 16, [3], 0),
    ("bf16", 2, 40, 9, 3, 72, 32, [2, 31], 36), ("f32", 2, 18, 12, 4, 64, 16, [0, 15], 24),
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norms", [True, False])
@pytest.mark.parametrize("io,B,N,H,G,P,page,lens,R", CASES)
def test_rope_against_fp64(io, B, N, H, G, P, page, lens, R, norms, interleaved):
    _check(_case(N * 7 + H, io, B, N, H, G, P, page, lens, R, norms=norms, interleaved=interleaved))


@pytest.mark.parametrize("kind", ["chain", "line", "star", "binary"])
@pytest.mark.parametrize("N", [1, 16, 31, 64, 200])
def test_rope_trees(kind, N):
    _check(_case(N, "bf16", 2, N, 4, 2, 64, 16, [7, 48], 64, tree=kind))


@pytest.mark.parametrize("io,N", [("bf16", 1000), ("f32", 257), ("bf16", 2049)])
def test_rope_prompts(io, N):
    _check(_case(N, io, 2, N, 2, 1, 64, 32, [0, 21], 64, tree="chain", interleaved=True, scale=0.75))


def test_rope_far_positions():
    """A cache whose tokens are 65536 to a row: angles of positions beyond what 32 bits hold to a fraction of a turn."""
    _check(_case(3, "f32", 2, 3, 2, 1, 8, 256, [1000003, 65535], 8, tree="chain"))


def test_rope_large_and_small_values_and_eps():
    c = _case(5, "f32", 2, 5, 2, 1, 64, 16, [3, 30], 64)
    c["rows"][0] *= 1e15
    c["rows"][1] *= 1e-12                                   # (the norm's eps decides)
    _check(c, eps=1e-20)
    c["rows"][1] = 0
    _check(c, eps=1e-6)


def test_rope_bad_sequences_leave_the_cache():
    """Bad trees, lengths and pages next to good ones: zeros, status, nothing appended; far page numbers are not followed."""
    c = _case(9, "bf16", 6, 20, 4, 2, 64, 16, [30, 31, 32, 5, -7, 12], 64, width=4)
    c["parent"][0, 7] = 7
    c["parent"][1, 0] = 0
    c["table"][2, 2] = 10 ** 9
    c["table"][3, 0] = -5
    c["lens"][5] = 45                                        # 45 + 20 tokens do not fit 4 pages of 16
    _check(c)


def test_rope_in_place_and_dense():
    """Dense q, k, v of their own; q_out = q."""
    c = _case(12, "bf16", 2, 19, 8, 2, 128, 16, [40, 3], 128)
    q, k, v = (np.ascontiguousarray(a) for a in _split(c["rows"], 8, 2, 128))
    want, wk, wv, _ = _run(c)
    o = lambda a: dev("bf16", a)  # noqa: E731
    qd, kc, vc = o(q), o(c["k"]), o(c["v"])
    got = st.stree_tree_rope(o(c["parent"]), o(c["lens"]), qd, o(k), o(v), kc, vc, o(c["table"]), o(c["turns"]), o(c["qn"]), o(c["kn"]), out=qd)
    assert got.data_ptr() == qd.data_ptr() and np.array_equal(host(got), want)
    assert np.array_equal(host(kc), wk, equal_nan=True) and np.array_equal(host(vc), wv, equal_nan=True)


def test_rope_odd_alignment():
    """Rows that start two bytes off a 16-byte boundary and lie an odd number of elements apart: the same values."""
    import torch
    c = _case(14, "bf16", 2, 21, 4, 2, 64, 16, [33, 2], 64)
    want, wk, wv, _ = _run(c)
    wide = torch.zeros(2, 21, 8 * 64 + 3, dtype=torch.bfloat16, device="cuda")
    wide[..., 1:-2] = dev("bf16", c["rows"])
    q, k, v = _split(wide[..., 1:-2], 4, 2, 64)
    kc, vc = dev("bf16", c["k"]), dev("bf16", c["v"])
    got = st.stree_tree_rope(dev("", c["parent"]), dev("", c["lens"]), q, k, v, kc, vc, dev("", c["table"]), dev("", c["turns"]),
                             dev("bf16", c["qn"]), dev("bf16", c["kn"]))
    fine = 64 * HALF["f32"]                                  # (another order of the norm's sum, then a rounding)
    within(host(got), want.astype(np.float64), (2 * HALF["bf16"] + fine) * np.abs(want) + fine, "q")
    assert np.array_equal(host(vc), wv, equal_nan=True)
