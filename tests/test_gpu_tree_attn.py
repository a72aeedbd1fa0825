"""stree_tree_attn against the fp64 form over paged caches whose unwritten slots hold NaN."""
import numpy as np
import pytest

from kv_helpers import HALF, attn_bound, caches, dev, host, rounded, tables, trees, within
from oracle import paged
from paper_2505_14969_amd import binding as st

pytestmark = pytest.mark.gpu


def _case(seed, io, N, H, G, P, page, lens, tree="random", width=None):
    rng = np.random.default_rng(seed)
    B, lens = len(lens), np.array(lens, np.int32)
    table, npages = tables(rng, lens, N, page, width=width)
    k, v = caches(rng, io, lens, N, table, npages, G, P, page)
    return dict(io=io, parent=trees(rng, B, N, tree), lens=lens, q=rounded(io, rng.standard_normal((B, N, H, P))), k=k, v=v, table=table)


def _run(c, plain=False, **more):
    import torch
    o = lambda a: None if a is None else dev(c["io"], a)  # noqa: E731
    status = torch.full((len(c["lens"]),), 77, dtype=torch.int32, device="cuda")
    got = st.stree_tree_attn(o(c["parent"]), o(c["lens"]), o(c["q"]), o(c["k"]), o(c["v"]), o(c["table"]), status=status, plain=plain, **more)
    return host(got), host(status)


def _want(c, scale=None):
    P = c["q"].shape[-1]
    return paged.attn(c["parent"], c["lens"], c["q"], c["k"], c["v"], c["table"], P ** -0.5 if scale is None else scale)


def _check(c, scale=None, plain=(False, True)):
    want, status, weight, score = _want(c, scale)
    bound = attn_bound(c["io"], want, weight, score, c["q"].shape[-1], int(c["lens"].max()) + c["q"].shape[1])
    for p in plain:
        got, gs = _run(c, plain=p, scale=scale)
        assert np.array_equal(gs, status), p
        within(got, want, bound, f"attention (plain {p})")


CASES = [
    # io, N, H, G, P, page, lengths
    ("bf16", 1, 8, 2, 128, 16, [0]), ("bf16", 1, 8, 2, 128, 16, [1, 15, 16, 31, 32, 33, 500]), ("f32", 1, 8, 2, 128, 16, [0, 3, 700]),
    ("bf16", 1, 16, 1, 64, 64, [1000, 63, 64]), ("bf16", 1, 4, 4, 64, 16, [257]), ("f32", 1, 3, 1, 64, 32, [129, 0]),
    ("bf16", 2, 6, 2, 128, 16, [30, 31]), ("bf16", 15, 8, 2, 128, 16, [100, 0, 17]), ("f32", 15, 4, 1, 64, 16, [33, 5]),
    ("bf16", 16, 4, 4, 128, 32, [64]), ("bf16", 17, 4, 1, 128, 16, [47]), ("bf16", 33, 6, 2, 64, 128, [127, 300]),
    ("bf16", 64, 8, 2, 128, 16, [200, 63]), ("f32", 64, 2, 1, 128, 16, [70]), ("bf16", 100, 4, 2, 128, 64, [513]),
    ("bf16", 256, 2, 1, 64, 16, [100]), ("f32", 130, 2, 2, 64, 256, [40]), ("bf16", 5, 8, 1, 256, 16, [90, 16]), ("f32", 7, 2, 1, 256, 16, [90]),
    ("bf16", 9, 4, 2, 80, 16, [77]), ("bf16", 30, 2, 1, 96, 32, [200]), ("bf16", 3, 4, 2, 8, 16, [50]), ("f32", 3, 4, 2, 4, 16, [50]),
    ("bf16", 4, 2, 1, 20, 16, [40]), ("f32", 4, 2, 1, 33, 16, [40]), ("bf16", 2, 2, 1, 1, 16, [20]), ("bf16", 12, 3, 3, 200, 16, [130]),
    ("bf16", 1, 40, 1, 128, 16, [300]), ("bf16", 1, 71, 1, 64, 16, [300]), ("bf16", 40, 5, 1, 128, 16, [95]), ("f32", 1, 20, 1, 64, 16, [1100]),
    ("bf16", 1, 128, 1, 64, 16, [400, 1]), ("bf16", 50, 16, 2, 64, 16, [333]), ("bf16", 3, 32, 8, 128, 16, [60, -1, 1, 700]),
]


@pytest.mark.parametrize("io,N,H,G,P,page,lens", CASES)
def test_attention_against_fp64(io, N, H, G, P, page, lens):
    _check(_case(N + H + P, io, N, H, G, P, page, lens))


@pytest.mark.parametrize("kind", ["chain", "line", "star", "binary"])
@pytest.mark.parametrize("io,N", [("bf16", 16), ("bf16", 63), ("f32", 40), ("bf16", 129)])
def test_attention_trees(kind, io, N):
    _check(_case(N, io, N, 4, 2, 64, 16, [0, 50], tree=kind))


@pytest.mark.parametrize("io,N,len0", [("bf16", 300, 1), ("bf16", 513, 700), ("f32", 270, 33)])
def test_attention_prompts(io, N, len0):
    _check(_case(N, io, N, 2, 1, 64, 32, [len0, 0], tree="chain"), plain=(False,))


@pytest.mark.parametrize("io,H,G,P,lens", [("bf16", 8, 2, 128, [9000, 12, 4097]), ("f32", 4, 1, 64, [5000, 2047]), ("bf16", 2, 1, 64, [20000])])
def test_attention_long(io, H, G, P, lens):
    """Split over workgroups and joined, sequences of very different lengths in one call."""
    _check(_case(H, io, 1, H, G, P, 16, lens))
    _check(_case(H, io, 6, H, G, P, 64, lens), plain=(False,))


def test_attention_wide_table_of_short_sequences():
    """A table made for far longer sequences than there are: the split goes by the lengths on the device."""
    c = _case(3, "bf16", 3, 8, 2, 128, 16, [40, 0, 333], width=4096)
    _check(c)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.01, 1.0, -0.5])
def test_attention_scales_and_peaks(io, scale):
    """Scores from flat to one that takes all, of both signs."""
    c = _case(8, io, 20, 4, 2, 128, 16, [300, 17])
    c["q"] = rounded(io, c["q"] * 3)
    _check(c, scale=scale)


def test_attention_infinities_and_nan_stay_on_their_paths():
    """A node whose key or value is not finite spoils the nodes that see it and no others; text that is not finite all."""
    for io in ("bf16", "f32"):
        for plain in (False, True):
            c = _case(21, io, 40, 4, 2, 128, 16, [100, 33])
            page, b, n = 16, 0, 100
            for node, what, value in ((7, "k", np.nan), (9, "v", np.nan), (11, "v", np.inf)):
                t = n + node
                pg = c["table"][b, t // page]
                if what == "k":
                    c["k"][pg, 1, t % page, 5] = value
                else:
                    c["v"][pg, 1, 3, t % page] = value
            got, status = _run(c, plain=plain)
            with np.errstate(invalid="ignore"):
                want, ws, weight, score = _want(c)
            assert np.array_equal(status, ws)
            inside = np.isfinite(want)
            assert np.array_equal(np.isfinite(got), inside), (io, plain)
            assert np.array_equal(np.isnan(got), np.isnan(want)), (io, plain)
            assert not inside[0].all() and inside[0, 0].all() and inside[1].all()
            score = np.where(np.isfinite(score), score, 0)
            bound = attn_bound(io, want, weight, score, 128, 200)
            assert np.all((np.abs(got - want) <= bound)[inside])
            # the text: everything of that head
            pg = c["table"][1, 0]
            c["v"][pg, 0, 4, 3] = np.nan
            got, _ = _run(c, plain=plain)
            assert np.isnan(got[1, :, :2, 4]).all() and np.isfinite(got[1, :, 2:]).all() and np.isfinite(got[1, :, :2, 5]).all()


def test_attention_bad_sequences():
    """Bad trees, lengths and pages next to good ones: zeros and a status; far page numbers are not followed."""
    for N, lens in ((20, [30, 31, 632, 5, -7, 12, 700]), (1, [30, 31, 632, 5, -7, 12, 700])):
        c = _case(9, "bf16", N, 8, 2, 64, 16, lens, width=45)
        if N > 1:
            c["parent"][0, 7] = 7
        c["parent"][1, 0] = 0
        c["table"][2, 39] = 10 ** 9
        c["table"][3, 0] = -5
        c["lens"][5] = 45 * 16 - N + 1
        c["table"][6, 2] = len(c["k"])
        _check(c)


def test_attention_strided_q_and_misaligned_rows():
    import torch
    c = _case(31, "bf16", 21, 8, 2, 128, 16, [90, 5])
    want, _, weight, score = _want(c)
    bound = attn_bound("bf16", want, weight, score, 128, 120)
    o = lambda a: dev("bf16", a)  # noqa: E731
    for pad, at in ((16, 8), (3, 1)):
        wide = torch.full((2, 21, 8 * 128 + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[..., at:at + 1024] = o(c["q"]).flatten(2)
        got = st.stree_tree_attn(o(c["parent"]), o(c["lens"]), wide[..., at:at + 1024].unflatten(2, (8, 128)), o(c["k"]), o(c["v"]), o(c["table"]))
        within(host(got), want, bound, f"q at {at}")


def test_attention_workspace_of_ones_own():
    """Scratch of the stated size, full of NaN, used again and again; one byte less is refused."""
    import torch
    c = _case(41, "bf16", 2, 8, 2, 128, 16, [3000, 100])
    o = lambda a: dev("bf16", a)  # noqa: E731
    t = [o(c[x]) for x in ("parent", "lens", "q", "k", "v", "table")]
    need = st.stree_attn_workspace(t[2], t[3], t[4], t[5])
    want, _ = _run(c)
    w = torch.full((max(need, 16) // 4 + 4,), float("nan"), device="cuda")
    for _ in range(3):
        got = st.stree_tree_attn(*t, workspace=w.view(torch.uint8)[:need])
        assert np.array_equal(host(got), want)
    assert torch.isnan(w[need // 4:]).all()
    if need:
        with pytest.raises(st.StreeError):
            st.stree_tree_attn(*t, workspace=w.view(torch.uint8)[:need - 1])


def test_attention_same_result_twice():
    c = _case(51, "bf16", 10, 8, 2, 128, 16, [5000, 1, 300])
    a, _ = _run(c)
    b, _ = _run(c)
    assert np.array_equal(a, b)
