"""stree_commit_kv whose new lengths take the place of an argument: of the accepted nodes too, which every workgroup of a sequence reads."""
import ctypes as C

import numpy as np
import pytest

from kv_helpers import caches, dev, host, tables, trees
from oracle import paged
from paper_2505_14969_amd import binding as st
from test_kv_refusals import _attn, _kv, lib  # noqa: F401

ALIAS = 6
AT = 0x10000000                                               # never dereferenced: the calls fail before


@pytest.mark.parametrize("off", [4, -4])
def test_lengths_that_lie_across_the_accepted_nodes_are_refused(lib, off):  # noqa: F811
    call = lambda accepted, lengths, out: lib.stree_commit_kv(C.byref(_attn()), C.byref(_kv()), AT, accepted, lengths, out, None, None)  # noqa: E731
    far = AT + 0x8000000
    assert call(far, AT, far + off) == ALIAS and call(AT, far, far + off) == ALIAS


@pytest.mark.gpu
@pytest.mark.parametrize("place", ["accepted", "lengths"])
@pytest.mark.parametrize("N", [20, 100])
def test_lengths_take_an_arguments_place(place, N):
    rng = np.random.default_rng(N)
    B, layers, G, P, page = 70, 5, 3, 64, 16
    lens = rng.integers(0, 60, B).astype(np.int32)
    lens[::9] = -1
    table, npages = tables(rng, lens, N, page)
    parent = trees(rng, B, N)
    accepted = rng.integers(-1, N, B).astype(np.int32)
    kv = [caches(rng, "bf16", lens, N, table, npages, G, P, page) for _ in range(layers)]
    k, v = (np.stack([x[i] for x in kv]) for i in range(2))
    kd, vd, ad, ld = dev("bf16", k), dev("bf16", v), dev("bf16", accepted), dev("bf16", lens)
    out = ad if place == "accepted" else ld
    got = st.stree_commit_kv(dev("bf16", parent), ad, ld, kd, vd, dev("bf16", table), lengths_out=out)
    want, _ = paged.commit(parent, accepted, lens, N, k, v, table)
    assert got.data_ptr() == out.data_ptr() and np.array_equal(host(got), want)
    assert np.array_equal(host(kd), k, equal_nan=True) and np.array_equal(host(vd), v, equal_nan=True)
