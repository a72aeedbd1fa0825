"""What the attention layers' entry points refuse before anything is launched, on the CPU: through the C ABI and through the
binding, and that no argument is lost on its way to the native half; the rotary frequencies, which are host data."""
import ctypes as C
import inspect
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2505_14969_amd import binding as st

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, I32 = torch.bfloat16, torch.int32
B, N, H, G, P, PAGE, M, NPAGES, R, L, F = 2, 6, 8, 2, 64, 16, 4, 9, 32, 3, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(st.LIB_PATH):
        from paper_2505_14969_amd import build
        build.build()
    return st.load()


# ------------------------------------------------------------------------------------------------ C ABI

NULL, ARG, SHAPE, DTYPE, STRIDE, ALIAS = None, 1, 2, 3, 4, 6
AT = 0x10000000                                               # never dereferenced: every call fails before


def _kv(**more):
    f = dict(nlayers=1, npages=NPAGES, page=PAGE, max_pages=M, nheads_kv=G, headdim=P, io_dtype=1, reserved=0, k=AT, v=AT, table=AT)
    return st.StreeKv(**{**f, **more})


def _attn(**more):
    f = dict(batch=B, nnodes=N, nheads=H, flags=0, rotary_dim=R, eps=1e-6, rope_scale=1.0, softmax_scale=0.0)
    return st.StreeAttn(**{**f, **more})


KV_BAD = [({"io_dtype": 7}, DTYPE), ({"npages": 0}, SHAPE), ({"page": 8}, SHAPE), ({"page": 24}, SHAPE), ({"page": 512}, SHAPE), ({"max_pages": 0}, SHAPE),
          ({"max_pages": (1 << 26) + 1}, SHAPE), ({"nheads_kv": 0}, SHAPE), ({"headdim": 0}, SHAPE), ({"headdim": 257}, SHAPE), ({"nlayers": 0}, SHAPE)]
NODES_BAD = [({"batch": -1}, SHAPE), ({"batch": 65536}, SHAPE), ({"nnodes": 0}, SHAPE), ({"nnodes": 257}, SHAPE)]
HEADS_BAD = [({"nheads": 7}, SHAPE), ({"nheads": 0}, SHAPE)]


def _rope(lib, a=None, kv=None, parent=AT, lengths=AT, q=AT, k=AT, v=AT, turns=AT, out=AT + 0x8000000, **_):
    return lib.stree_tree_rope(C.byref(_attn(**(a or {}))), C.byref(_kv(**(kv or {}))), parent, lengths, q, k, v, None, None, turns, out, None, None)


def _att(lib, a=None, kv=None, parent=AT, lengths=AT, q=AT, out=AT + 0x8000000, w=AT, n=1 << 40):
    return lib.stree_tree_attn(C.byref(_attn(**(a or {}))), C.byref(_kv(**(kv or {}))), parent, lengths, q, out, None, w, n, None)


def _commit(lib, a=None, kv=None, parent=AT, accepted=AT, lengths=AT, out=AT + 0x8000000):
    return lib.stree_commit_kv(C.byref(_attn(**(a or {}))), C.byref(_kv(**(kv or {}))), parent, accepted, lengths, out, None, None)


def _pool(**more):
    return C.byref(st.StreePool(**{**dict(held=AT, refs=AT, free=AT, nfree=AT), **more}))


def _resize(lib, kv=None, pool=None, batch=B, tokens=AT):
    return lib.stree_resize_kv(C.byref(_kv(**(kv or {}))), _pool(**(pool or {})), batch, tokens, None, None)


def _fork(lib, kv=None, pool=None, batch=B, forks=F, src=AT, dst=AT, lengths=AT, status=AT):
    return lib.stree_fork_kv(C.byref(_kv(**(kv or {}))), _pool(**(pool or {})), batch, forks, src, dst, lengths, status, None)


@pytest.mark.parametrize("N,heads", [(1, 8), (16, 8), (64, 32), (2048, 32), (1 << 18, 8)])
def test_scratch_does_not_grow_with_the_batch(lib, N, heads):
    """Parts of rows that were cut: as many as the chip holds at once, whatever the number of sequences."""
    need = [lib.stree_attn_workspace_bytes(C.byref(_attn(batch=b, nnodes=N, nheads=heads)), C.byref(_kv(nheads_kv=8, headdim=128, max_pages=1 << 14)))
            for b in (8, 64, 256)]
    units = [8 * 8, 64 * 8, 256 * 8]
    assert need[0] == 0 or [n - 8 * u for n, u in zip(need, units)] == [need[0] - 8 * units[0]] * 3
    assert max(need) <= 2 * 512 * 256 * (128 + 2) * 4 + 8 * units[2] + 32


def test_abi_refusals(lib):
    for call in (_rope, _att, _commit, _resize, _fork):
        for kv, rc in KV_BAD:
            assert call(lib, kv=kv) == rc, (call.__name__, kv)
        assert call(lib, kv={"table": None}) == ARG
    for call in (_rope, _att, _commit):
        for a, rc in NODES_BAD:
            assert call(lib, a=a) == rc, (call.__name__, a)
        assert call(lib, a={"batch": 0}) == 0                   # (nothing to do)
        assert call(lib, parent=NULL, a={"nnodes": (1 << 24) + 1}) == SHAPE
        assert call(lib, lengths=NULL) == ARG and call(lib, kv={"k": None}) == ARG and call(lib, kv={"v": None}) == ARG
    for call in (_rope, _att):
        for a, rc in HEADS_BAD:
            assert call(lib, a=a) == rc
        assert call(lib, kv={"nlayers": 2}) == SHAPE
        assert call(lib, parent=NULL, a={"batch": 256, "nnodes": 1 << 23}) == SHAPE      # batch * nodes * heads from 2^31 on
        assert call(lib, a={"q_stride_n": H * P - 1}) == STRIDE and call(lib, a={"q_stride_n": -H * P}) == STRIDE
        assert call(lib, a={"q_stride_n": 1 << 60}) == STRIDE and call(lib, a={"q_stride_n": 1 << 56}) == STRIDE
        assert call(lib, q=NULL) == ARG and call(lib, out=NULL) == ARG
        rows = B * N * H * P * 2
        for q in (AT + 0x8000000 + 2, AT + 0x8000000 - rows + 2, AT + 0x8000000 + rows - 2):
            assert call(lib, q=q) == ALIAS
        assert call(lib, q=AT + 0x8000000, a={"q_stride_n": H * P + 8}) == ALIAS         # (in place, but not the same rows)
    assert _att(lib, q=AT + 0x8000000) == ALIAS
    assert _rope(lib, k=AT + 0x8000000) == ALIAS and _rope(lib, v=AT + 0x8000000 + 64) == ALIAS
    assert _rope(lib, a={"k_stride_n": G * P - 1}) == STRIDE and _rope(lib, a={"v_stride_n": 1}) == STRIDE
    for r in (-2, 31, P + 2):
        assert _rope(lib, a={"rotary_dim": r}) == SHAPE
    assert _rope(lib, a={"eps": -1.0}) == SHAPE and _rope(lib, a={"eps": float("nan")}) == SHAPE
    assert _rope(lib, turns=NULL) == ARG and _rope(lib, k=NULL) == ARG and _rope(lib, v=NULL) == ARG
    assert _att(lib, a={"softmax_scale": float("inf")}) == SHAPE and _att(lib, a={"softmax_scale": float("nan")}) == SHAPE
    assert lib.stree_attn_workspace_bytes(C.byref(_attn()), C.byref(_kv(page=17))) == C.c_size_t(-1).value
    assert lib.stree_attn_workspace_bytes(C.byref(_attn(batch=0)), C.byref(_kv())) == 0
    assert lib.stree_attn_workspace_bytes(None, None) == C.c_size_t(-1).value
    assert _commit(lib, accepted=NULL) == ARG and _commit(lib, out=NULL) == ARG
    assert _commit(lib, out=AT + 4) == ALIAS and _commit(lib, out=AT - 4) == ALIAS
    assert _resize(lib, tokens=NULL) == ARG and _resize(lib, batch=-1) == SHAPE and _resize(lib, batch=4097) == SHAPE
    assert _resize(lib, batch=0) == 0 and _resize(lib, kv={"max_pages": 1 << 26}, batch=16) == SHAPE
    for name in ("held", "refs", "free", "nfree"):
        assert _resize(lib, pool={name: None}) == ARG and _fork(lib, pool={name: None}) == ARG
    assert _fork(lib, forks=-1) == SHAPE and _fork(lib, forks=4097) == SHAPE and _fork(lib, forks=0) == 0
    for name in ("src", "dst", "lengths", "status"):
        assert _fork(lib, **{name: None}) == ARG


def test_structs_match_the_header(tmp_path):
    both = {"stree_kv": st.StreeKv, "stree_attn": st.StreeAttn, "stree_pool": st.StreePool}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "%s"' % os.path.join(ROOT, "include", "stree.h"), "int main(void) {"]
    want = []
    for name, cls in both.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(C.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field))
            want.append(getattr(cls, field).offset)
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-o", str(tmp_path / "l"), str(tmp_path / "l.c")], check=True)
    assert [int(x) for x in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.split()] == want


# ------------------------------------------------------------------------------------------------ frequencies

def test_frequencies():
    two_pi = 2 * math.pi
    j = np.arange(32)
    plain = 10000.0 ** (-2 * j / 64) / two_pi
    get = lambda *a, **k: st.stree_rope_frequencies(*a, device="cpu", **k).numpy()  # noqa: E731
    near = lambda a, b: np.testing.assert_allclose(a, b, rtol=1e-14)  # noqa: E731
    near(get(64), plain)
    near(get(64, scaling="linear", factor=4.0), plain / 4)
    stretched = get(64, scaling="base", factor=4.0)
    near(stretched[0], plain[0])
    near(stretched[-1], plain[-1] / 4)
    near(get(2, scaling="base", factor=4.0), [1 / two_pi])
    ramp = get(64, base=500000.0, scaling="ramp", factor=8.0, low=1.0, high=4.0, original=8192.0)
    f = 500000.0 ** (-2 * j / 64) / two_pi
    fast, slow = f * 8192 >= 4, f * 8192 <= 1
    near(ramp[fast], f[fast])
    near(ramp[slow], f[slow] / 8)
    middle = ~fast & ~slow
    assert middle.any() and (ramp[middle] < f[middle]).all() and (ramp[middle] > f[middle] / 8).all()
    assert get(0).shape == (0,)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=-2), dict(rotary_dim=258), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, base=float("inf")),
                dict(rotary_dim=8, scaling="linear", factor=0.5), dict(rotary_dim=8, scaling="ramp", factor=2.0, low=4.0, high=4.0),
                dict(rotary_dim=8, scaling="ramp", factor=2.0, original=0.0), dict(rotary_dim=8, scaling="base", factor=float("nan"))):
        with pytest.raises(st.StreeError):
            st.stree_rope_frequencies(device="cpu", **bad)
    with pytest.raises(KeyError):
        st.stree_rope_frequencies(8, scaling="other", device="cpu")


# ------------------------------------------------------------------------------------------------ binding

def _good():
    z, o = torch.zeros, lambda *s: torch.zeros(*s, dtype=I32)  # noqa: E731
    k, v = z(NPAGES, G, PAGE, P, dtype=BF), z(NPAGES, G, P, PAGE, dtype=BF)
    nodes = dict(parent=o(B, N), lengths=o(B))
    cache = dict(k_cache=k, v_cache=v, table=o(B, M))
    layers = dict(k_cache=z(L, NPAGES, G, PAGE, P, dtype=BF), v_cache=z(L, NPAGES, G, P, PAGE, dtype=BF))
    pool = dict(held=o(B), table=o(B, M), refs=o(NPAGES), free=o(NPAGES), nfree=o(1))
    return {
        "stree_tree_rope": dict(**nodes, q=z(B, N, H, P, dtype=BF), k=z(B, N, G, P, dtype=BF), v=z(B, N, G, P, dtype=BF), **cache,
                                turns=z(R // 2, dtype=torch.float64), q_norm=z(P, dtype=BF), k_norm=z(P, dtype=BF)),
        "stree_tree_attn": dict(**nodes, q=z(B, N, H, P, dtype=BF), **cache),
        "stree_attn_workspace": dict(q=z(B, N, H, P, dtype=BF), **cache),
        "stree_commit_kv": dict(**nodes, accepted=o(B), table=o(B, M), **layers),
        "stree_resize_kv": dict(tokens=o(B), **pool, page=PAGE),
        "stree_fork_kv": dict(src=o(F), dst=o(F), lengths=o(B), **pool, **layers),
    }


def _strided(t):
    return torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)[..., :t.shape[-1]]


COMMON = [("table", lambda t: t[0], ValueError), ("table", lambda t: t.long(), AssertionError), ("table", _strided, AssertionError),
          ("lengths", lambda t: t[:-1], AssertionError), ("lengths", lambda t: t.long(), AssertionError)]
CACHE = [("k_cache", lambda t: t[0, 0], ValueError), ("k_cache", lambda t: t.half(), (TypeError, AssertionError)), ("v_cache", lambda t: t.float(), AssertionError),
         ("v_cache", lambda t: t.transpose(-1, -2), AssertionError), ("v_cache", _strided, AssertionError), ("k_cache", _strided, AssertionError)]
NODES = [("parent", lambda t: t[:, :-1], AssertionError), ("parent", lambda t: t.long(), AssertionError), ("status", lambda t: torch.zeros(B), AssertionError),
         ("status", lambda t: torch.zeros(B + 1, dtype=I32), AssertionError), ("table", lambda t: t[:-1], AssertionError)]
POOL = [("held", lambda t: t[:-1], AssertionError), ("refs", lambda t: t[:-1], AssertionError), ("free", lambda t: t.long(), AssertionError),
        ("nfree", lambda t: torch.zeros(2, dtype=I32), AssertionError)]
REFUSED = [("stree_tree_rope", *c) for c in COMMON + CACHE + NODES] + [("stree_tree_attn", *c) for c in COMMON + CACHE + NODES]
REFUSED += [("stree_commit_kv", *c) for c in COMMON + CACHE + NODES] + [("stree_fork_kv", *c) for c in COMMON + CACHE + POOL]
REFUSED += [("stree_resize_kv", *c) for c in COMMON[:3] + POOL]
REFUSED += [
    ("stree_tree_rope", "q", lambda t: t[0], ValueError), ("stree_tree_rope", "q", lambda t: t.float(), AssertionError), ("stree_tree_rope", "q", _strided, AssertionError),
    ("stree_tree_rope", "q", lambda t: t.numpy(force=True) if t.dtype != BF else np.zeros(t.shape), (TypeError, AttributeError)),
    ("stree_tree_rope", "k", lambda t: t[:, :, :1], AssertionError), ("stree_tree_rope", "v", lambda t: t.float(), AssertionError), ("stree_tree_rope", "v", _strided, AssertionError),
    ("stree_tree_rope", "q", lambda t: t[:, :1].expand(B, N, H, P), AssertionError),      # rows that lie on one another
    ("stree_tree_rope", "k", lambda t: t[:1, :1].expand(B, N, G, P), AssertionError), ("stree_tree_attn", "q", lambda t: t[:1, :1].expand(B, N, H, P), AssertionError),
    ("stree_tree_rope", "turns", lambda t: t.float(), AssertionError), ("stree_tree_rope", "turns", lambda t: torch.zeros(P, dtype=torch.float64), AssertionError),
    ("stree_tree_rope", "q_norm", lambda t: t[:-1], AssertionError), ("stree_tree_rope", "k_norm", lambda t: t.float(), AssertionError),
    ("stree_tree_rope", "out", lambda t: torch.zeros(B, N, H, P), AssertionError), ("stree_tree_rope", "out", lambda t: torch.zeros(B, N, H, 2 * P, dtype=BF)[..., :P], AssertionError),
    ("stree_tree_rope", "eps", lambda v: "small", TypeError), ("stree_tree_rope", "k_cache", lambda t: t[None], ValueError),
    ("stree_tree_attn", "q", lambda t: t[..., :-1], AssertionError), ("stree_tree_attn", "q", lambda t: t[0], ValueError), ("stree_tree_attn", "scale", lambda v: 0.0, AssertionError),
    ("stree_tree_attn", "out", lambda t: torch.zeros(B, N, H + 1, P, dtype=BF), AssertionError), ("stree_tree_attn", "scale", lambda v: "big", TypeError),
    ("stree_attn_workspace", "q", lambda t: t[0], ValueError), ("stree_attn_workspace", "q", lambda t: t[:, :, :-1], ValueError),
    ("stree_commit_kv", "accepted", lambda t: t[:-1], AssertionError), ("stree_commit_kv", "lengths_out", lambda t: torch.zeros(B), AssertionError),
    ("stree_commit_kv", "parent", lambda t: None, TypeError),                             # (a chain says how long it is)
    ("stree_resize_kv", "tokens", lambda t: t[:-1], AssertionError), ("stree_resize_kv", "page", lambda v: 2 ** 31, AssertionError),
    ("stree_resize_kv", "page", lambda v: 1.5, TypeError), ("stree_resize_kv", "refs", lambda t: t[None], ValueError),
    ("stree_fork_kv", "dst", lambda t: t[:-1], AssertionError), ("stree_fork_kv", "src", lambda t: t[None], ValueError), ("stree_fork_kv", "status", lambda t: torch.zeros(F), AssertionError),
]


@pytest.mark.parametrize("name,arg,change,error", REFUSED)
def test_binding_refuses_before_anything_is_launched(name, arg, change, error):
    call = _good()[name]
    call[arg] = change(call.get(arg))
    with pytest.raises(error) as e:
        getattr(st, name)(**call)
    assert "GPU" not in str(e.value) or error is AttributeError


@pytest.mark.parametrize("name", sorted(set(_good()) - {"stree_attn_workspace"}))
def test_tensors_that_are_not_on_the_gpu(name):
    with pytest.raises(AssertionError, match="tensors on one GPU"):
        getattr(st, name)(**_good()[name])


def test_every_argument_reaches_the_native_half():
    with open(os.path.join(ROOT, "paper_2505_14969_amd", "csrc", "host_kv.hpp")) as f:
        text = f.read()

    class Seen:
        def __getattr__(self, entry):
            return lambda *args: args
    kept, st._host = st._native(), Seen()
    try:
        seen = []
        for name, function, count in re.findall(r'METHOD\("(\w+)", (\w+), (\d+)\)', text):
            names = re.findall(r"\w+", re.search(r"PyObject \*%s\(const Args &a\) \{\s*enum \{([^}]*)\}" % function, text).group(1))
            f = getattr(st, "stree_" + name)
            assert list(f(**{n: n for n in inspect.signature(f).parameters})) == names and len(names) == int(count), name
            seen.append("stree_" + name)
        assert sorted(seen) == sorted(_good())
    finally:
        st._host = kept
