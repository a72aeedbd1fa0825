"""Inputs of the tests of the attention layers: paged caches whose unwritten slots hold NaN, tables in random order."""
from __future__ import annotations

import numpy as np

from paper_2505_14969_amd import synth

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}              # half a step of a rounding, relative to the value


def rounded(io, a):
    a = np.asarray(a, np.float32)
    return synth.round_to_bf16(a) if io == "bf16" else a


def dev(io, a):
    """fp32 numpy (exact in io, NaN kept) -> cuda tensor of the storage type."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    if a.dtype == np.int32 or a.dtype == np.float64:
        return t.cuda()
    return t.to(torch.bfloat16 if io == "bf16" else torch.float32).cuda()


def host(t):
    import torch
    return t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()


def trees(rng, B, N, kind="random"):
    if kind == "chain":
        return None
    p = np.zeros((B, N), np.int32)
    for b in range(B):
        for i in range(N):
            p[b, i] = -1 if i == 0 else {"random": rng.integers(max(0, i - 8), i), "line": i - 1, "star": 0,
                                         "binary": (i - 1) // 2}[kind]
    return p


def tables(rng, lens, N, page, spare=2, width=None):
    """Table rows of random pages for len + N tokens (-1 behind them) and the number of pages of the pool."""
    need = [0 if n < 0 else -(-(n + N) // page) for n in lens]
    width = width or max(max(need), 1)
    npages = sum(need) + spare
    order = rng.permutation(npages).astype(np.int32)
    table = np.full((len(lens), width), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, npages


def caches(rng, io, lens, extra, table, npages, G, P, page):
    """Keys and values of the first len + extra tokens of each sequence; NaN everywhere else."""
    k = np.full((npages, G, page, P), np.nan, np.float32)
    v = np.full((npages, G, P, page), np.nan, np.float32)
    for b, n in enumerate(lens):
        t = np.arange(max(n, 0) + extra if n >= 0 else 0)
        pg = table[b, t // page]
        k[pg, :, t % page] = rounded(io, rng.standard_normal((len(t), G, P)))
        v[pg, :, :, t % page] = rounded(io, rng.standard_normal((len(t), G, P)))
    return k, v


def within(got, want, bound, what):
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    off = np.where(np.isnan(want), 0.0, np.abs(got.astype(np.float64) - want) - bound)
    worst = np.unravel_index(np.argmax(off), off.shape)
    assert off.max() <= 0, f"{what}: {got[worst]} for {want[worst]} at {worst}, {off.max():.3e} over the bound"


def attn_bound(io, want, weight, score, P, keys):
    """Rounding of the result; of the probabilities (bf16 operands) above and below the fraction line, as far as they
    weigh; and fp32 sums of P products in the scores (an error of a score is a relative one of its probability) and of
    `keys` terms in the results, all at their worst."""
    p = HALF["bf16"] if io == "bf16" else 0.0
    s = (P + 8) * HALF["f32"] * score[..., None] + 8 * HALF["f32"]
    return HALF[io] * np.abs(want) * (1 + 2 * p) + 2 * (p + s + keys * HALF["f32"]) * weight + 1e-30
