"""stree_commit_kv, stree_resize_kv and stree_fork_kv against the plain forms: all of the caches, tables and pools, bit for bit."""
import numpy as np
import pytest

from kv_helpers import dev, host, rounded, tables, trees
from oracle import paged
from paper_2505_14969_amd import binding as st

pytestmark = pytest.mark.gpu


def _filled(rng, io, layers, npages, G, P, page):
    k = rounded(io, rng.standard_normal((layers, npages, G, page, P)))
    v = rounded(io, rng.standard_normal((layers, npages, G, P, page)))
    return k, v


def _commit(seed, io, N, G, P, page, lens, accepted, layers=2, tree="random", width=None, spoil=None, inplace=False):
    import torch
    rng = np.random.default_rng(seed)
    lens, accepted = np.array(lens, np.int32), np.array(accepted, np.int32)
    B = len(lens)
    table, npages = tables(rng, lens, N, page, width=width)
    k, v = _filled(rng, io, layers, npages, G, P, page)
    parent = trees(rng, B, N, tree)
    if spoil:
        spoil(parent, table, lens)
    o = lambda a: None if a is None else dev(io, a)  # noqa: E731
    kd, vd, ld = o(k), o(v), o(lens)
    status = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    one = layers == 1
    got = st.stree_commit_kv(o(parent), o(accepted), ld, kd[0] if one else kd, vd[0] if one else vd, o(table),
                             lengths_out=ld if inplace else None, status=status, nnodes=N)
    want, ws = paged.commit(parent, accepted, lens, N, k, v, table)
    assert np.array_equal(host(got), want) and np.array_equal(host(status), ws)
    assert (got.data_ptr() == ld.data_ptr()) == inplace and (inplace or np.array_equal(host(ld), lens))
    assert np.array_equal(host(kd), k) and np.array_equal(host(vd), v)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("io,N,G,P,page,lens,accepted,layers", [
    ("bf16", 1, 8, 128, 16, [0], [0], 1), ("bf16", 15, 8, 128, 16, [100], [14], 3), ("f32", 15, 2, 64, 32, [31, 0], [7, -1], 2),
    ("bf16", 64, 2, 128, 16, [5, 16, 47], [63, 30, 0], 1), ("bf16", 256, 1, 64, 16, [9, 700], [255, 254], 2), ("f32", 49, 3, 33, 16, [3], [48], 1),
    ("bf16", 40, 2, 7, 16, [15, -1], [39, 12], 2), ("bf16", 17, 1, 256, 64, [60], [16], 1), ("f32", 100, 2, 4, 256, [250], [99], 1),
    ("bf16", 30, 5, 80, 128, [127], [29], 2), ("bf16", 12, 2, 8, 16, [14], [11], 1)])
def test_commit_moves_the_path(io, N, G, P, page, lens, accepted, layers, inplace):
    _commit(N, io, N, G, P, page, lens, accepted, layers=layers, inplace=inplace)


@pytest.mark.parametrize("kind", ["chain", "line", "star", "binary"])
@pytest.mark.parametrize("N", [2, 63, 200])
def test_commit_trees(kind, N):
    for inplace in (False, True):
        _commit(N, "bf16", N, 2, 64, 16, [37, 0], [N - 1, N // 2], tree=kind, inplace=inplace)


def test_commit_prompt_and_bad_sequences():
    _commit(1, "bf16", 1000, 1, 64, 16, [3, 0, -1], [999, 1000, 4], tree="chain")

    def spoil(parent, table, lens):
        parent[0, 3] = 9
        table[2, 1] = 1 << 30
        table[3, 0] = -1
        lens[4] = 100
    for inplace in (False, True):
        _commit(2, "bf16", 20, 2, 64, 16, [1, 2, 3, 30, 5, 6], [19, 20, 19, 19, 19, -2], spoil=spoil, width=4, inplace=inplace)


def _pool(rng, B, M, npages, lens, page, shared=()):
    """Sequences with the pages of their lengths; `shared`: (row, row it shares full pages with)."""
    order = rng.permutation(npages).astype(np.int32)
    table, held, refs = np.full((B, M), -1, np.int32), np.zeros(B, np.int32), np.zeros(npages, np.int32)
    at = 0
    for b, n in enumerate(lens):
        held[b] = -(-max(n, 0) // page)
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    for b, other in shared:
        table[b, :held[b]] = table[other, :held[b]]
    for b in range(B):
        np.add.at(refs, table[b, :held[b]], 1)
    taken = refs > 0
    rest = np.array([p for p in order if not taken[p]], np.int32)
    free = np.zeros(npages, np.int32)
    free[:len(rest)] = rest
    return dict(table=table, held=held, refs=refs, free=free, nfree=np.array([len(rest)], np.int32))


NAMES = ("held", "table", "refs", "free", "nfree")


def _resize(pool, tokens, page):
    import torch
    tokens = np.array(tokens, np.int32)
    d = {n: dev("", pool[n]) for n in NAMES}
    status = torch.full((len(tokens),), 77, dtype=torch.int32, device="cuda")
    got = st.stree_resize_kv(dev("", tokens), *(d[n] for n in NAMES), page, status=status)
    assert got is d["held"]
    want = paged.resize(tokens, *(pool[n] for n in NAMES), page)
    assert np.array_equal(host(status), want), (host(status), want)
    for n in NAMES:
        assert np.array_equal(host(d[n]), pool[n]), n


@pytest.mark.parametrize("B,M,npages,page,seed", [(1, 1, 1, 16, 0), (4, 8, 40, 16, 1), (64, 40, 1500, 32, 2), (1100, 6, 4000, 16, 3), (4096, 3, 9000, 64, 4),
                                                  (3, 3000, 9000, 16, 5)])
def test_resize_random(B, M, npages, page, seed):
    """Rows that grow and shrink at once, with pages shared by several rows and too few of them."""
    rng = np.random.default_rng(seed)
    for few in (False, True):
        lens = rng.integers(0, M * page + 1, B)
        while -(-lens // page).sum() > npages:
            lens = lens // 2
        shared = [(b, rng.integers(0, b)) for b in range(1, B) if rng.random() < 0.3]
        shared = [(b, o) for b, o in shared if -(-lens[b] // page) <= -(-lens[o] // page)]
        pool = _pool(rng, B, M, npages, lens, page, shared)
        if few:
            pool["nfree"][0] = min(pool["nfree"][0], 2)
        for _ in range(3):
            tokens = rng.integers(-1, M * page + 1, B)
            _resize(pool, tokens, page)
        _resize(pool, [0] * B, page)
        assert not pool["refs"].any() and not pool["held"].any() and (few or pool["nfree"][0] == npages)


def test_resize_refuses_what_contradicts_itself():
    rng = np.random.default_rng(7)
    pool = _pool(rng, 6, 8, 40, [50, 60, 70, 80, 20, 0], 16)
    pool["table"][0, 1] = 1000                              # outside the pool
    pool["table"][1, 0] = -3
    pool["refs"][pool["table"][2, 0]] = 0                   # held by nobody
    pool["held"][3] = 9
    pool["table"][4, 1] = pool["table"][4, 0]               # twice in a row, held once
    _resize(pool, [0, 0, 0, 0, 0, 129], 16)
    _resize(pool, [16, 16, 16, 16, 16, 16], 16)
    pool["nfree"][0] = 41
    _resize(pool, [0] * 6, 16)
    pool["nfree"][0] = -1
    _resize(pool, [0] * 6, 16)
    pool = _pool(rng, 2, 4, 10, [0, 16], 16)
    pool["free"][pool["nfree"][0] - 1] = 99                 # a damaged stack
    _resize(pool, [30, 16], 16)


def _fork(pool, lens, src, dst, k, v, io="bf16"):
    import torch
    src, dst = np.array(src, np.int32), np.array(dst, np.int32)
    d = {n: dev("", pool[n]) for n in NAMES}
    ld, kd, vd = dev("", lens), dev(io, k), dev(io, v)
    status = torch.full((len(src),), 77, dtype=torch.int32, device="cuda")
    got = st.stree_fork_kv(dev("", src), dev("", dst), ld, *(d[n] for n in NAMES), kd, vd, status=status)
    want = paged.fork(src, dst, lens, *(pool[n] for n in NAMES), k, v)
    assert got is status and np.array_equal(host(status), want), (host(status), want)
    for n in NAMES:
        assert np.array_equal(host(d[n]), pool[n]), n
    assert np.array_equal(host(ld), lens) and np.array_equal(host(kd), k) and np.array_equal(host(vd), v)


@pytest.mark.parametrize("io,G,P,page,layers", [("bf16", 8, 128, 16, 3), ("f32", 2, 64, 32, 1), ("bf16", 1, 1, 16, 2), ("f32", 3, 33, 128, 2)])
def test_fork_shares_and_copies(io, G, P, page, layers):
    rng = np.random.default_rng(P)
    lens = np.array([3 * page + 5, 2 * page, 0, page - 1, 0, 0, 0, 0, -1], np.int32)
    pool = _pool(rng, 9, 6, 30, lens, page)
    k, v = _filled(rng, io, layers, 30, G, P, page)
    _fork(pool, lens, [0, 0, 1, 3], [4, 5, 6, 7], k, v, io)
    assert pool["refs"].max() == 3
    _resize(pool, [-1, -1, -1, -1, 0, 0, 0, 0, 0], page)
    _fork(pool, lens, [2, 3, 3], [4, 2, 6], k, v, io)       # (2: of length 0, source and target at once)


def test_fork_refusals():
    page = 16
    rng = np.random.default_rng(3)
    lens = np.array([40, 33, 20, 50, 16, 0, 0, 0, 0, -1, 0, 0], np.int32)
    pool = _pool(rng, 12, 6, 30, lens, page)
    k, v = _filled(rng, "bf16", 2, 30, 2, 64, page)
    pool["table"][1, 1] = 77
    pool["refs"][pool["table"][2, 1]] = 0
    lens[3] = 65                                            # beyond its pages
    _fork(pool, lens, [0, 1, 2, 3, 9, 0, 0, -1, 12, 0, 0, 4, 4], [5, 6, 6, 6, 6, 5, 0, 6, 6, -1, 12, 6, 6], k, v)
    pool["nfree"][0] = 1                                    # one page for two forks; one that needs none
    lens2 = np.array([40, 33, 20, 50, 16, 0, 0, 0, 0, -1, 0, 0], np.int32)
    pool2 = _pool(rng, 12, 6, 30, lens2, page)
    pool2["nfree"][0] = 1
    _fork(pool2, lens2, [0, 0, 4, 0], [5, 6, 7, 8], k, v)
    pool2["nfree"][0] = 31
    _fork(pool2, lens2, [0], [8], k, v)
    pool2["nfree"][0] = 3
    pool2["free"][2] = -9
    _fork(pool2, lens2, [0, 0], [8, 10], k, v)


def test_many_forks():
    page, F = 16, 2000
    rng = np.random.default_rng(4)
    lens = np.concatenate((rng.integers(0, 60, 50), np.zeros(F))).astype(np.int32)
    pool = _pool(rng, 50 + F, 5, 200 + F, lens, page)
    k, v = _filled(rng, "bf16", 1, 200 + F, 1, 8, page)
    _fork(pool, lens, rng.integers(0, 50, F), 50 + rng.permutation(F), k, v)
