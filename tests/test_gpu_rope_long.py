"""stree_tree_rope on long prompts: the page numbers of all of a prompt's slots are looked at before anything is written, by a number of
workgroups that does not grow with the prompt."""
import numpy as np
import pytest

from kv_helpers import host
from paper_2505_14969_amd import binding as st

pytestmark = pytest.mark.gpu


def _tensors(n, P, io="bf16", H=1, G=1, B=1, page=16, first=0):
    import torch
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(n + P)
    width = (first + n) // page + 1
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    table = torch.randperm(B * width, generator=g, device="cuda").to(torch.int32).view(B, width)
    cache = torch.zeros(B * width, G, page, P, dtype=dt, device="cuda"), torch.zeros(B * width, G, P, page, dtype=dt, device="cuda")
    turns = st.stree_rope_frequencies(P // 2 * 2)
    return (torch.full((B,), first, dtype=torch.int32, device="cuda"), rand(B, n, H, P), rand(B, n, G, P), rand(B, n, G, P), *cache, table, turns)


@pytest.mark.parametrize("P", [16, 7])
def test_time_grows_with_the_prompt_and_not_with_its_square(P):
    """Eight times the tokens: at most 20 times as long (64 if every workgroup's look at the table grew along)."""
    import torch
    took = []
    for n in (1 << 17, 1 << 20):
        t = _tensors(n, P)
        call = lambda: st.stree_tree_rope(None, *t)  # noqa: E731
        call()
        torch.cuda.synchronize()
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            call()
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        took.append(min(times))
        print(f"{n} tokens of {P}: {took[-1]:.3f} ms", flush=True)
    assert took[1] < 20 * took[0]


@pytest.mark.parametrize("io,n,H,G,P,first", [("bf16", 70000, 2, 1, 64, 13), ("f32", 33333, 3, 1, 24, 0), ("bf16", 70001, 1, 1, 7, 5), ("f32", 5000, 1, 1, 33, 40)])
def test_long_prompts_piece_by_piece(io, n, H, G, P, first):
    """A long prompt in one call gives what its pieces of 2000 tokens give; a bad page anywhere leaves everything as it was."""
    import torch
    B = 2
    lens, q, k, v, kc, vc, table, turns = _tensors(n, P, io, H, G, B, first=first)
    status = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    got = st.stree_tree_rope(None, lens, q, k, v, kc, vc, table, turns, status=status)
    assert not status.any()
    kp, vp = torch.zeros_like(kc), torch.zeros_like(vc)
    for at in range(0, n, 2000):
        piece = [x[:, at:at + 2000].contiguous() for x in (q, k, v)]
        out = st.stree_tree_rope(None, lens + at, *piece, kp, vp, table, turns)
        assert torch.equal(out, got[:, at:at + 2000]), at
    assert torch.equal(kc, kp) and torch.equal(vc, vp)
    for entry in (first // 16, (first + n // 2) // 16, (first + n - 1) // 16):
        bad = table.clone()
        bad[1, entry] = -3
        k2, v2 = torch.zeros_like(kc), torch.zeros_like(vc)
        out = st.stree_tree_rope(None, lens, q, k, v, k2, v2, bad, turns, status=status)
        assert status.tolist() == [0, st.SEQ_PAGE] and not out[1].any() and torch.equal(out[0], got[0])
        assert not k2[table[1].long()].any() and not v2[table[1].long()].any()
        mine = table[0].long()
        assert torch.equal(k2[mine], kc[mine]) and torch.equal(v2[mine], vc[mine])


def test_long_prompt_in_place():
    lens, q, k, v, kc, vc, table, turns = _tensors(40000, 64, H=2)
    want = st.stree_tree_rope(None, lens, q, k, v, kc, vc, table, turns)
    out = st.stree_tree_rope(None, lens, q, k, v, kc, vc, table, turns, out=q)
    assert out.data_ptr() == q.data_ptr() and np.array_equal(host(out), host(want))
