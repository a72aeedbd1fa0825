"""stree_tree_rope: cosine and sine to the last bits of fp32, also where they pass zero."""
import numpy as np
import pytest

from paper_2505_14969_amd import binding as st

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("P,scale", [(64, 1.0), (30, 1.0), (128, 0.5)])
def test_cosine_and_sine_relative_to_themselves(P, scale, interleaved):
    """Rows of (1, 0) come out as (cos, sin).  Each is right relative to its own size: 4 units in the last place (2^-23) of the
    sine and cosine of the fraction in 32 bits, which may be twice as large as the result that the fraction's remaining bits make of it; half
    a unit for each of the two roundings behind them; and 2 pi times what the 64-bit product position x turns is off by."""
    import torch
    N, R = 3000, P
    base = 40000
    turns = np.array([0.37, 0.25, 1 / 3, 0.5000003, 0.0123, 0.1591549430918953, 0.49999, 1e-6])[np.arange(R // 2) % 8] * (1 + 1e-4 * np.arange(R // 2))
    first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    row = torch.zeros(P)
    row[first] = 1
    q = row.expand(1, N, 1, P).contiguous().cuda()
    pages = (base + N) // 256 + 1
    k_cache, v_cache = torch.zeros(1, 1, 256, P, device="cuda"), torch.zeros(1, 1, P, 256, device="cuda")
    table = torch.zeros(1, pages, dtype=torch.int32, device="cuda")      # (one page for all: only q is looked at)
    got = st.stree_tree_rope(None, torch.tensor([base], dtype=torch.int32).cuda(), q, q, q, k_cache, v_cache, table, torch.from_numpy(turns).cuda(),
                             interleaved=interleaved, rope_scale=scale)[0, :, 0].double().cpu().numpy()
    t = (base + np.arange(N))[:, None] * turns
    part = t - np.rint(t)
    # of the fraction of a turn: quadrants by hand, so that the values near zero keep all of their bits
    quarter = np.rint(4 * part).astype(int)
    x = 2 * np.pi * (part - quarter / 4)
    cos = np.choose(quarter % 4, [np.cos(x), -np.sin(x), -np.cos(x), np.sin(x)]) * scale
    sin = np.choose(quarter % 4, [np.sin(x), np.cos(x), -np.sin(x), -np.cos(x)]) * scale
    assert (np.abs(sin) < 0.05 * scale).sum() > 100 and (np.abs(cos) < 0.05 * scale).sum() > 100
    for name, value, want in (("cos", got[:, first], cos), ("sin", got[:, second], sin)):
        bound = (2 * 4 + 2 * 0.5) * 2.0 ** -23 * np.abs(want) + 2 * np.pi * scale * np.abs(t) * 2.0 ** -53
        off = np.abs(value - want) / bound
        assert off.max() <= 1, (name, off.max(), want[np.unravel_index(off.argmax(), off.shape)])
