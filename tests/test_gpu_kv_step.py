"""The attention layers' operators together, as a decoding loop uses them: several layers on one page table, trees of changing
size, accepted nodes, forks and rows given back, against the fp64 forms; captured into a graph and replayed; on another stream."""
import numpy as np
import pytest

from kv_helpers import HALF, attn_bound, dev, host, rounded, trees, within
from oracle import paged
from paper_2505_14969_amd import binding as st

pytestmark = pytest.mark.gpu

NAMES = ("held", "table", "refs", "free", "nfree")


def _pool(B, M, npages):
    import torch
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = dict(held=i32(B), table=i32(B, M) - 1, refs=i32(npages), free=torch.arange(npages, dtype=torch.int32, device="cuda"), nfree=i32(1) + npages)
    return pool


@pytest.mark.parametrize("io,G,R,P,page", [("bf16", 2, 4, 128, 16), ("f32", 1, 3, 64, 32), ("bf16", 3, 1, 80, 16)])
def test_decoding_loop(io, G, R, P, page):
    """Prompts, then trees: every layer's q, cache and attention, the pool and the lengths against the plain forms run beside
    them.  Two sequences, one of them forked in between and the fork dropped again; one row of the batch idle."""
    import torch
    rng = np.random.default_rng(P)
    H, B, M, npages, L = G * R, 4, 24, 60, 2
    turns = st.stree_rope_frequencies(P // 4 * 2, base=500000.0, scaling="ramp", factor=4.0, original=64.0)
    tn = turns.cpu().numpy()
    pool = _pool(B, M, npages)
    hp = {n: host(pool[n]).copy() for n in NAMES}
    k = np.full((L, npages, G, page, P), np.nan, np.float32)
    v = np.full((L, npages, G, P, page), np.nan, np.float32)
    kd, vd = dev(io, k), dev(io, v)
    lengths, hl = dev("", np.array([0, 0, -1, -1], np.int32)), np.array([0, 0, -1, -1], np.int32)
    qn, kn = rounded(io, rng.uniform(0.5, 1.5, P)), rounded(io, rng.uniform(0.5, 1.5, P))

    def resize(tokens):
        tokens = np.array(tokens, np.int32)
        st.stree_resize_kv(dev("", tokens), *(pool[n] for n in NAMES), page)
        paged.resize(tokens, *(hp[n] for n in NAMES), page)
        for n in NAMES:
            assert np.array_equal(host(pool[n]), hp[n]), n

    for N, kind, accept in ((21, "chain", [20, 20, -1, -1]), (15, "binary", [14, 9, -1, -1]), (1, "chain", [0, 0, -1, -1]), ("fork", None, None),
                            (33, "random", [30, 32, -1, 20]), (6, "star", [5, -1, -1, 3]), ("drop", None, None), (12, "line", [11, 4, -1, -1])):
        if N == "fork":
            src, dst = np.array([0], np.int32), np.array([3], np.int32)
            got = st.stree_fork_kv(dev("", src), dev("", dst), lengths, *(pool[n] for n in NAMES), kd, vd)
            before = [hp[n].copy() for n in NAMES]
            paged.fork(src, dst, hl, *(hp[n] for n in NAMES), k, v)
            assert not host(got).any() and np.array_equal(host(lengths), hl) and not np.array_equal(before[1], hp["table"])
            continue
        if N == "drop":
            resize([-1, -1, -1, 0])
            hl[3] = -1
            lengths[3] = -1
            continue
        resize([n + N if n >= 0 else -1 for n in hl])
        parent = trees(rng, B, N, kind)
        pd = None if parent is None else dev("", parent)
        for layer in range(L):
            rows = rounded(io, rng.standard_normal((B, N, (H + 2 * G) * P)))
            rd = dev(io, rows)
            cut = lambda a, i, j: a[..., i * P:j * P].reshape(B, N, j - i, P)  # noqa: E731
            q, kk, vv = cut(rows, 0, H), cut(rows, H, H + G), cut(rows, H + G, H + 2 * G)
            qd, kkd, vvd = (rd[..., i * P:j * P].unflatten(2, (j - i, P)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
            got_q = st.stree_tree_rope(pd, lengths, qd, kkd, vvd, kd[layer], vd[layer], pool["table"], turns, dev(io, qn), dev(io, kn))
            wk, wv = k[layer].astype(np.float64), v[layer].astype(np.float64)
            want_q, status, size_q, _ = paged.rope(parent, hl, q, kk, vv, wk, wv, hp["table"], tn, qn, kn, 1e-6, False, 1.0)
            assert not status.any()
            fine = (P / 2 + 24) * HALF["f32"]
            within(host(got_q), want_q, HALF[io] * (1 + fine) * np.abs(want_q) + fine * size_q, f"q of layer {layer}")
            # from here on the plain form goes on with what the kernels wrote, so that its inputs are theirs
            k[layer], v[layer] = host(kd[layer]), host(vd[layer])
            assert np.array_equal(np.isnan(k[layer]), np.isnan(wk)) and np.array_equal(v[layer], wv.astype(np.float32), equal_nan=True)
            got = st.stree_tree_attn(pd, lengths, got_q, kd[layer], vd[layer], pool["table"])
            want, status, weight, score = paged.attn(parent, hl, host(got_q), k[layer], v[layer], hp["table"], P ** -0.5)
            assert not status.any()
            within(host(got), want, attn_bound(io, want, weight, score, P, 200), f"attention of layer {layer}")
        accepted = np.array(accept, np.int32)
        out = st.stree_commit_kv(pd, dev("", accepted), lengths, kd, vd, pool["table"], lengths_out=lengths, nnodes=N)
        hl, _ = paged.commit(parent, accepted, hl, N, k, v, hp["table"])
        assert out is lengths and np.array_equal(host(lengths), hl)
        assert np.array_equal(host(kd), k, equal_nan=True) and np.array_equal(host(vd), v, equal_nan=True)
    resize([0, 0, 0, 0])
    assert host(pool["nfree"])[0] == npages


def _step_inputs(rng, B, N, H, G, P, page, M):
    import torch
    npages = B * M
    table = dev("", rng.permutation(npages).astype(np.int32).reshape(B, M))
    kd = torch.randn(1, npages, G, page, P, device="cuda").to(torch.bfloat16)
    vd = torch.randn(1, npages, G, P, page, device="cuda").to(torch.bfloat16)
    return table, kd, vd


def test_step_in_a_graph():
    """Rotation, attention and the commit in place captured once and replayed with other rows, trees and lengths: the same as
    the calls made one by one, with other work and synchronisation in between; two graphs of the same tensors in turn."""
    import torch
    rng = np.random.default_rng(1)
    B, N, H, G, P, page, M = 3, 20, 8, 2, 128, 16, 60
    table, k0, v0 = _step_inputs(rng, B, N, H, G, P, page, M)
    turns = st.stree_rope_frequencies(P)
    rows = torch.zeros(B, N, H + 2 * G, P, dtype=torch.bfloat16, device="cuda")
    parent, accepted = torch.zeros(B, N, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    lengths, status = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    kd, vd = k0.clone(), v0.clone()

    def step(lens, kc, vc):
        q = st.stree_tree_rope(parent, lens, rows[:, :, :H], rows[:, :, H:H + G], rows[:, :, H + G:], kc[0], vc[0], table, turns)
        out = st.stree_tree_attn(parent, lens, q, kc[0], vc[0], table, status=status)
        st.stree_commit_kv(parent, accepted, lens, kc, vc, table, lengths_out=lens)
        return out

    def draw():
        parent.copy_(dev("", trees(rng, B, N)))
        parent[:, 0] = -1
        rows.copy_(torch.randn(rows.shape, device="cuda"))
        accepted.copy_(dev("", rng.integers(-1, N, B).astype(np.int32)))

    draw()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(lengths.clone(), kd.clone(), vd.clone())
    side.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(lengths, kd, vd))
        graphs.append(g)
    kd.copy_(k0), vd.copy_(v0), lengths.copy_(dev("", np.array([700, 3, -1], np.int32)))
    ek, ev, el = kd.clone(), vd.clone(), lengths.clone()
    for i in range(6):
        draw()
        if i == 3:                                            # a bad tree and a bad page on the way
            parent[0, 5] = 5
        want = step(el, ek, ev).clone()
        want_status = status.clone()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], want) and torch.equal(lengths, el) and torch.equal(status, want_status), i
        assert torch.equal(kd, ek) and torch.equal(vd, ev), i
        assert bool(want_status[0] == 6) == (i == 3)
    assert int(el[2]) == -1 and int(el[0]) > 700


def test_calls_go_to_the_current_stream():
    """The work waits for what stands before it on the stream that is current, not on the default one."""
    import torch
    rng = np.random.default_rng(2)
    B, N, H, G, P, page, M = 2, 10, 8, 2, 64, 16, 20
    table, kd, vd = _step_inputs(rng, B, N, H, G, P, page, M)
    turns = st.stree_rope_frequencies(P)
    real = torch.randn(B, N, H + 2 * G, P, device="cuda").to(torch.bfloat16)
    lengths, parent = torch.full((B,), 250, dtype=torch.int32, device="cuda"), dev("", trees(rng, B, N))
    k2, v2 = kd.clone(), vd.clone()

    def step(rows, kc, vc):
        q = st.stree_tree_rope(parent, lengths, rows[:, :, :H], rows[:, :, H:H + G], rows[:, :, H + G:], kc[0], vc[0], table, turns)
        return st.stree_tree_attn(parent, lengths, q, kc[0], vc[0], table)
    want = step(real, kd, vd)
    torch.cuda.synchronize()
    big = torch.randn(4096, 4096, device="cuda")
    rows, stream = torch.zeros_like(real), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(10):
            big = big @ big * 1e-3                            # (keeps the stream busy before the rows are there)
        rows.copy_(real)
        got = step(rows, k2, v2)
    stream.synchronize()
    assert torch.equal(got, want) and torch.equal(k2, kd) and torch.equal(v2, vd)


def test_two_calls_at_once():
    """Calls on two streams, each with scratch of its own."""
    import torch
    rng = np.random.default_rng(3)
    table, kd, vd = _step_inputs(rng, 2, 1, 8, 2, 128, 16, 300)
    lengths = dev("", np.array([4700, 2000], np.int32))
    qs = [torch.randn(2, 1, 8, 128, device="cuda").to(torch.bfloat16) for _ in range(2)]
    want = [st.stree_tree_attn(None, lengths, q, kd[0], vd[0], table) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(st.stree_tree_attn(None, lengths, qs[i], kd[0], vd[0], table))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GB: pages at its end are found, by every operator."""
    import torch
    G, P, page = 8, 128, 256
    npages = 2 ** 32 // (G * P * page * 2) + 40               # bytes of K beyond 2^32, elements beyond 2^31
    kd = torch.zeros(1, npages, G, page, P, dtype=torch.bfloat16, device="cuda")
    vd = torch.zeros(1, npages, G, P, page, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(4)
    N, H, lens = 12, 16, np.array([250, 3], np.int32)
    table = np.array([[npages - 1, npages - 7], [npages - 3, 0]], np.int32)
    small = {int(p): i for i, p in enumerate(table.ravel())}
    parent = trees(rng, 2, N)
    for b in range(2):                                        # the text
        for t in range(lens[b]):
            pg = int(table[b, t // page])
            kd[0, pg, :, t % page] = torch.randn(G, P, device="cuda").to(torch.bfloat16)
            vd[0, pg, :, :, t % page] = torch.randn(G, P, device="cuda").to(torch.bfloat16)
    rows = torch.randn(2, N, H + 2 * G, P, device="cuda").to(torch.bfloat16)
    pd, ld, td = dev("", parent), dev("", lens), dev("", table)
    q = st.stree_tree_rope(pd, ld, rows[:, :, :H], rows[:, :, H:H + G], rows[:, :, H + G:], kd[0], vd[0], td, st.stree_rope_frequencies(P))
    got = host(st.stree_tree_attn(pd, ld, q, kd[0], vd[0], td))
    plain = host(st.stree_tree_attn(pd, ld, q, kd[0], vd[0], td, plain=True))
    pages = torch.tensor(sorted(small, key=small.get), device="cuda")
    k, v = host(kd[0, pages]), host(vd[0, pages])
    near = np.array([[small[int(p)] for p in row] for row in table], np.int32)
    want, _, weight, score = paged.attn(parent, lens, host(q), k, v, near, P ** -0.5)
    assert np.abs(k[0, :, 250:]).max() > 0                    # (the nodes' rows are there)
    for g in (got, plain):
        within(g, want, attn_bound("bf16", want, weight, score, P, 300), "far pages")
    accepted = dev("", np.array([N - 1, 5], np.int32))
    out = st.stree_commit_kv(pd, accepted, ld, kd, vd, td)
    k1, v1 = k[None].copy(), v[None].copy()
    wl, _ = paged.commit(parent, host(accepted), lens, N, k1, v1, near)
    assert np.array_equal(host(out), wl) and np.array_equal(host(kd[0, pages]), k1[0]) and np.array_equal(host(vd[0, pages]), v1[0])
    held = dev("", np.array([2, 2], np.int32))
    refs = torch.zeros(npages, dtype=torch.int32, device="cuda")
    refs[pages] = 1
    both = torch.cat((td, torch.full_like(td[:1], -1)))
    free, nfree = torch.zeros(npages, dtype=torch.int32, device="cuda"), dev("", np.array([1], np.int32))
    free[0] = npages - 20
    lens3 = torch.cat((out, out[:1] * 0))
    st3 = st.stree_fork_kv(dev("", np.array([0], np.int32)), dev("", np.array([2], np.int32)), lens3, torch.cat((held, held[:1] * 0)), both, refs, free,
                           nfree, kd, vd)
    assert int(st3[0]) == 0 and int(lens3[2]) == int(lens3[0])
    last = int(lens3[0]) // page
    assert int(both[2, last]) == npages - 20
    assert torch.equal(kd[0, npages - 20], kd[0, int(both[0, last])]) and torch.equal(vd[0, npages - 20], vd[0, int(both[0, last])])
