"""The attention layers' part of a decoding step, as cases that can be timed and compared.

In a hybrid model the token tree that the scan verifies also goes through attention layers, whose keys and values lie in a
paged cache.  A case is one pass of one of four kinds, through the binding's public calls:

  rope    ``stree_tree_rope``: norm of queries and keys, rotation, keys and values appended to the cache
  attn    ``stree_tree_attn``: attention of the tree's nodes over the cache and their ancestors (one node: a new token)
  commit  ``stree_commit_kv``: the accepted path's rows moved together, in every layer
  pages   a turn of the page tables of a search over branches: ``stree_resize_kv`` gives back what the last turn's
          branches held, ``stree_fork_kv`` makes new ones, ``stree_resize_kv`` takes pages for the next trees

Cache: keys [pages, heads, page, headdim], values [pages, heads, headdim, page] (tokens side by side), page numbers in a
table row per sequence.  Sizes are those of generic attention layers (32 query heads on 8 of 128 channels and others);
trees those of this library's other cases (15, 49 and 64 nodes).
"""
import math

import numpy as np
import torch

own = False
_binding = None

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _st():
    global _binding
    if _binding is None:
        from paper_2505_14969_amd import binding
        _binding = binding
    return _binding


# ------------------------------------------------------------------------------------------------------------- cases

def _case(kind, batch, length, nodes=1, heads=32, kv_heads=8, headdim=128, page=16, dtype="bf16", tree="random", ragged=False,
          layers=1, **more):
    return dict(kind=kind, batch=batch, length=length, nodes=nodes, heads=heads, kv_heads=kv_heads, headdim=headdim, page=page,
                dtype=dtype, tree=tree, ragged=ragged, layers=layers, **more)


def _rope(batch, length, rotary=128, interleaved=False, norm=True, scaling="none", **more):
    return _case("rope", batch, length, rotary=rotary, interleaved=interleaved, norm=norm, scaling=scaling, **more)


def listed():
    return [
        # one user's next token at a far position: launch and latency
        _rope(1, 20011, name="rope_b1_n1"),
        # a serving batch of 64-node trees, frequencies stretched for long contexts
        _rope(16, 2000, nodes=64, ragged=True, scaling="ramp", name="rope_b16_n64"),
        # two prompts of odd length in fp32, pairs side by side, half of the head rotated, no norm
        _rope(2, 0, nodes=2047, tree="chain", dtype="f32", rotary=64, interleaved=True, norm=False, name="rope_b2_t2047_f32"),
        # one user, a small draft tree in fp32, as a model is checked: launches and host time count
        _case("attn", 1, 500, nodes=15, dtype="f32", name="attn_b1_n15_f32"),
        # one user, one new token behind a very long text: little to do but stream the cache
        _case("attn", 1, 131071, page=64, name="attn_b1_n1_l131071"),
        # a full serving batch, one new token each, lengths all different
        _case("attn", 64, 4096, ragged=True, name="attn_b64_n1"),
        # the benchmark's trees (16 sequences of 64 nodes) behind contexts of different lengths
        _case("attn", 16, 4096, nodes=64, ragged=True, name="attn_b16_n64"),
        # a piece of a long prompt: every token sees the cache and what stands before it in the piece
        _case("attn", 2, 1537, nodes=512, tree="chain", page=64, name="attn_b2_t512"),
        # one user, one layer, a small tree
        _case("commit", 1, 700, nodes=15, name="commit_b1_n15"),
        # a full batch, beams of 3 x 16 tokens, eight layers at once
        _case("commit", 64, 300, nodes=49, ragged=True, layers=8, name="commit_b64_n49"),
        # two texts, three branches each
        _case("pages", 2, 777, nodes=16, branches=3, layers=4, ragged=True, name="pages_b2"),
        # sixteen texts with three branches each, eight layers
        _case("pages", 16, 1000, nodes=49, page=32, branches=3, layers=8, ragged=True, name="pages_b16"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    """A case of the ranges above: 1 to 64 sequences, 1 to 256 nodes (or a prompt), contexts of 1 to 131072 tokens."""
    kind = rng.choice(("rope", "attn", "attn", "attn", "commit", "pages"))
    heads, kv_heads, headdim = rng.choice(((32, 8, 128), (32, 8, 128), (40, 8, 128), (64, 8, 128), (24, 24, 64), (32, 4, 64),
                                           (12, 2, 64), (28, 4, 128), (16, 4, 80), (16, 1, 256)))
    page = rng.choice((16, 16, 32, 64, 128))
    shape = dict(heads=heads, kv_heads=kv_heads, headdim=headdim, page=page, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")),
                 ragged=rng.random() < 0.6)
    width = kv_heads * headdim
    batch = _log_uniform(rng, 1, 64)
    if kind == "rope":
        chain = rng.random() < 0.3
        nodes = _log_uniform(rng, 1, 4096 if chain else 256)
        batch = max(1, min(batch, 8192 // nodes, 8192 * 48 * 128 // (nodes * (heads + 2 * kv_heads) * headdim)))
        length = _log_uniform(rng, 1, 100000)
        batch = max(1, min(batch, 2 ** 26 // (width * (length + nodes))))
        rotary = rng.choice((headdim, headdim, headdim // 2))
        return _rope(batch, length, rotary=rotary, interleaved=rng.random() < 0.4, norm=rng.random() < 0.7,
                     scaling=rng.choice(("none", "linear", "base", "ramp")), nodes=nodes, tree="chain" if chain else "random", **shape)
    if kind == "attn":
        chain = rng.random() < 0.15
        nodes = _log_uniform(rng, 16, 1024) if chain else rng.choice((1, 1, 0)) or _log_uniform(rng, 2, 256)
        batch = max(1, min(batch, 1024 // nodes))
        # no more cache rows, scores or products than the largest listed cases have
        most = min(2 ** 28 // (batch * width), 2 ** 27 // (batch * heads * nodes), 2 ** 34 // (batch * heads * nodes * headdim)) - nodes
        return _case("attn", batch, _log_uniform(rng, 1, max(1, min(131071, most))), nodes=nodes, tree="chain" if chain else "random", **shape)
    if kind == "commit":
        nodes, layers = _log_uniform(rng, 2, 256), rng.randint(1, 8)
        batch = max(1, min(batch, 3136 // nodes))
        length = _log_uniform(rng, 1, 2000)
        return _case("commit", max(1, min(batch, 2 ** 28 // (width * layers * (length + nodes)))), length, nodes=nodes, layers=layers, **shape)
    branches, layers = rng.randint(1, 4), rng.randint(1, 8)
    nodes, length = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 1000)
    batch = max(1, min(_log_uniform(rng, 1, 16), 48 // branches, 2 ** 24 // (width * layers * page * branches),
                       2 ** 28 // (width * layers * (length + page + (branches + 1) * (nodes + 2 * page)))))
    return _case("pages", batch, length, nodes=nodes, branches=branches, layers=layers, **shape)


# ------------------------------------------------------------------------------------------------------------ inputs

def _lengths(c):
    """Tokens that the cache holds of each sequence: all alike, or from a quarter of the length on."""
    if not c["ragged"]:
        return [c["length"]] * c["batch"]
    return [max(1, int(c["length"] * (0.25 + 0.75 * ((b * 0.6180339887 + 0.99) % 1.0)))) for b in range(c["batch"])]


def _turns(c):
    """Turns a position of each pair, for a context stretched eight times from 8192 tokens."""
    r, factor = c["rotary"], 8.0
    base = 10000.0 * (factor ** (r / (r - 2)) if c["scaling"] == "base" and r > 2 else 1.0)
    t = base ** (-2.0 * np.arange(r // 2) / r) / (2 * math.pi)
    if c["scaling"] == "linear":
        t = t / factor
    if c["scaling"] == "ramp":
        keep = np.clip((8192 * t - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        t = t * (keep + (1 - keep) / factor)
    return torch.from_numpy(t).cuda()


def _parents(rng, c):
    """Random trees whose nodes hang on one of the eight before them; None for a chain."""
    if c["tree"] == "chain":
        return None
    i = np.arange(c["nodes"])
    p = i - 1 - (rng.random((c["batch"], c["nodes"])) * np.minimum(np.maximum(i, 1), 8)).astype(np.int64)
    p[:, 0] = -1
    return torch.from_numpy(p.astype(np.int32)).cuda()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    io = DTYPES[c["dtype"]]
    B, N, H, G, P, page, layers = (c[k] for k in ("batch", "nodes", "heads", "kv_heads", "headdim", "page", "layers"))
    lens = _lengths(c)
    reach = max(lens) + N
    width = -(-reach // page)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=io)  # noqa: E731
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()  # noqa: E731
    s = {"case": c, "reach": reach}
    if c["kind"] == "pages":
        F = B * c["branches"]
        held = [-(-(n + N) // page) for n in lens]
        npages = sum(held) + c["branches"] * sum(-(-(n + N) // page) - n // page for n in lens) + 5
        order = torch.randperm(npages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B + F, width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b in range(B):
            table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
        refs = torch.zeros(npages, dtype=torch.int32, device="cuda")
        refs[order[:at].long()] = 1
        free = torch.zeros(npages, dtype=torch.int32, device="cuda")
        free[:npages - at] = order[at:]
        s.update(table=table, refs=refs, free=free, nfree=i32([npages - at]), held=i32(held + [0] * F), lengths=i32(lens + [0] * F),
                 kept=i32(lens + [0] * F), wanted=i32([n + N for n in lens] + [lens[f // c["branches"]] + N for f in range(F)]),
                 src=i32([f // c["branches"] for f in range(F)]), dst=i32(list(range(B, B + F))))
    else:
        npages = sum(-(-(n + N) // page) for n in lens) + 3
        order = torch.randperm(npages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b in range(B):
            n = -(-(lens[b] + N) // page)
            table[b, :n] = order[at:at + n]
            at += n
        s.update(table=table, lengths=i32(lens), parent=_parents(rng, c))
    many = (layers, npages) if c["kind"] in ("commit", "pages") else (npages,)
    s.update(k_cache=rand(*many, G, page, P), v_cache=rand(*many, G, P, page))
    if c["kind"] == "rope":
        # the projection's output: queries, keys and values as column ranges of one row
        rows = rand(B, N, (H + 2 * G) * P)
        s.update(q=rows[..., :H * P].unflatten(2, (H, P)), k=rows[..., H * P:(H + G) * P].unflatten(2, (G, P)),
                 v=rows[..., (H + G) * P:].unflatten(2, (G, P)), turns=_turns(c), q_norm=None, k_norm=None)
        if c["norm"]:
            s.update(q_norm=rand(P) * 0.1 + 1, k_norm=rand(P) * 0.1 + 1)
    if c["kind"] == "attn":
        s.update(q=rand(B, N, H, P))
    if c["kind"] == "commit":
        # three of four sequences accept a node, drawn from all
        s.update(accepted=i32(np.where(np.arange(B) % 4 == 3, -1, rng.integers(N // 2, N, B))))
    return s


# ------------------------------------------------------------------------------------------------------- plain forms

def _ancestors(parent, batch, nodes, device):
    """[B,N,N]: whether node j lies on the path of node i (the tree's mask), by repeated products."""
    if parent is None:
        return torch.ones(nodes, nodes, dtype=torch.bool, device=device).tril().expand(batch, nodes, nodes)
    i = torch.arange(nodes, device=device)
    reach = ((parent.long()[:, :, None] == i) | (i[:, None] == i)).float()
    for _ in range(max(1, (nodes - 1).bit_length())):
        reach = (reach @ reach).clamp(max=1)
    return reach > 0


def _rope_plain(s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    B, N = q.shape[:2]
    R, page = c["rotary"], c["page"]
    if s["parent"] is None:
        depth = torch.arange(N, device=q.device).expand(B, N)
    else:
        depth = _ancestors(s["parent"], B, N, q.device).sum(2) - 1
    lengths = s["lengths"].long()
    angle = ((lengths[:, None] + depth).double()[:, :, None] * s["turns"]).frac() * (2 * math.pi)   # far positions: 64 bits
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        y = x.clone()
        u, w = (slice(0, R, 2), slice(1, R, 2)) if c["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        y[..., u] = x[..., u] * cos - x[..., w] * sin
        y[..., w] = x[..., u] * sin + x[..., w] * cos
        return y.to(q.dtype)

    slot = lengths[:, None] + torch.arange(N, device=q.device)
    at = s["table"].long().gather(1, slot // page)
    s["k_cache"][at, :, slot % page] = turned(k, s["k_norm"])
    s["v_cache"][at, :, :, slot % page] = v
    return {"q": turned(q, s["q_norm"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attn_plain(s):
    c, q = s["case"], s["q"]
    B, N, H, P = q.shape
    G, page = c["kv_heads"], c["page"]
    lengths = s["lengths"].long()
    slot = torch.arange(s["reach"], device=q.device)
    at = s["table"].long()[:, slot // page].clamp(min=0)
    K = s["k_cache"][at, :, slot % page].float()                     # [B, L, G, P]
    V = s["v_cache"][at, :, :, slot % page].float()
    Q = q.float().view(B, N, G, H // G, P).permute(0, 2, 1, 3, 4).reshape(B, G, -1, P)
    score = Q @ K.permute(0, 2, 3, 1).contiguous() / math.sqrt(P)
    node = slot - lengths[:, None]                                   # which of the tree's nodes a slot holds
    seen = _ancestors(s["parent"], B, N, q.device).gather(2, node.clamp(0, N - 1)[:, None].expand(B, N, -1))
    seen = (seen & (node < N)[:, None]) | (node < 0)[:, None]
    score = score.view(B, G, N, H // G, -1).masked_fill(~seen[:, None, :, None], -math.inf)
    weight = (score - score.amax(-1, keepdim=True)).exp()
    weight = weight / weight.sum(-1, keepdim=True)
    out = weight.view(B, G, N * (H // G), -1) @ V.permute(0, 2, 1, 3).contiguous()
    return out.view(B, G, N, H // G, P).permute(0, 2, 1, 3, 4).reshape(B, N, H, P).to(q.dtype)


def _commit_plain(s):
    c, lengths, accepted = s["case"], s["lengths"].long(), s["accepted"].long()
    B, N, page = c["batch"], c["nodes"], c["page"]
    node = torch.arange(N, device=lengths.device).expand(B, N)
    path = _ancestors(s["parent"], B, N, lengths.device).gather(1, accepted.clamp(min=0)[:, None, None].expand(B, 1, N))[:, 0]
    path = path & (accepted >= 0)[:, None]
    count = path.sum(1)
    source = torch.where(path, node, node + N).argsort(1)            # the path's nodes first, in order
    source = torch.where(node < count[:, None], source, node)        # (behind them every row stays)
    take, put = lengths[:, None] + source, lengths[:, None] + node
    table = s["table"].long()
    src, dst = table.gather(1, take // page), table.gather(1, put // page)
    rows, cols = s["k_cache"][:, src, :, take % page], s["v_cache"][:, src, :, :, take % page]
    for i in range(c["layers"]):
        s["k_cache"][i][dst, :, put % page] = rows[:, :, i]
        s["v_cache"][i][dst, :, :, put % page] = cols[:, :, i]
    return {"lengths": (lengths + count).int(), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _resize_plain(tokens, held, table, refs, free, nfree, page):
    n, far = refs.numel(), table.numel()
    j = torch.arange(table.shape[1], device=table.device)
    need = torch.where(tokens < 0, held, (tokens + page - 1) // page)
    drop = (j >= need[:, None]) & (j < held[:, None])
    number = torch.where(drop, table, n).long().view(-1)
    less = torch.zeros(n + 1, dtype=torch.int32, device=table.device).index_add_(0, number, torch.ones_like(number, dtype=torch.int32))[:n]
    refs -= less
    gone = (less > 0) & (refs == 0)
    first = torch.full((n + 1,), far, device=table.device).scatter_reduce_(0, number, torch.arange(far, device=table.device), "amin")[:n]
    rank = torch.arange(n, device=table.device)
    freed = torch.where(gone, first, far + rank).argsort()           # pages in the order in which they were dropped first
    stack = torch.cat((free, free.new_zeros(1)))
    stack[torch.where(rank < gone.sum(), nfree + rank, n)] = freed.int()
    free.copy_(stack[:n])
    nfree += gone.sum().int()
    table.masked_fill_(drop, -1)
    more = (need - held).clamp(min=0)
    before = more.cumsum(0) - more
    more = torch.where(before + more <= nfree, more, 0)
    grown = (j >= held[:, None]) & (j < (held + more)[:, None])
    page_of = free[(nfree - 1 - before[:, None] - j + held[:, None]).clamp(0, n - 1).long()]
    table.copy_(torch.where(grown, page_of, table))
    refs.copy_(torch.cat((refs, refs.new_zeros(1))).index_fill_(0, torch.where(grown, page_of, n).long().view(-1), 1)[:n])
    nfree -= more.sum().int()
    held.copy_(torch.minimum(held, need) + more)


def _fork_plain(src, dst, lengths, held, table, refs, free, nfree, k_cache, v_cache):
    page, src, dst = v_cache.shape[-1], src.long(), dst.long()
    length = lengths[src]
    full, part = length // page, (length % page > 0).int()
    fresh = free[(nfree - part.cumsum(0)).clamp(min=0).long()]
    j = torch.arange(table.shape[1], device=table.device)
    rows = table[src]
    shared = j < full[:, None]
    refs += torch.zeros(refs.numel() + 1, dtype=torch.int32, device=table.device).index_add_(
        0, torch.where(shared, rows, refs.numel()).long().view(-1), torch.ones_like(rows).view(-1))[:-1]
    last = (j == full[:, None]) & (part > 0)[:, None]
    table[dst] = torch.where(shared, rows, torch.where(last, fresh[:, None], -1))
    refs.copy_(torch.cat((refs, refs.new_zeros(1))).index_fill_(0, torch.where(part > 0, fresh, refs.numel()).long(), 1)[:-1])
    held[dst] = full + part
    lengths[dst] = length
    nfree -= part.sum().int()
    # (a fork without a partial page copies its first page onto itself)
    take = rows.gather(1, torch.where(part > 0, full, 0).long()[:, None])[:, 0]
    put = torch.where(part > 0, fresh, take).long()
    k_cache[:, put] = k_cache[:, take.long()]
    v_cache[:, put] = v_cache[:, take.long()]


def _pages(s, resize, fork):
    pool = s["refs"], s["free"], s["nfree"]
    page = s["case"]["page"]
    resize(s["kept"], s["held"], s["table"], *pool, page)
    fork(s["src"], s["dst"], s["lengths"], s["held"], s["table"], *pool, s["k_cache"], s["v_cache"])
    resize(s["wanted"], s["held"], s["table"], *pool, page)
    return {k: s[k] for k in ("table", "held", "lengths", "refs", "free", "nfree", "k_cache", "v_cache")}


def run(state):
    s, c = state, state["case"]
    if not own:
        if c["kind"] == "pages":
            return _pages(s, _resize_plain, _fork_plain)
        return {"rope": _rope_plain, "attn": _attn_plain, "commit": _commit_plain}[c["kind"]](s)
    st = _st()
    if c["kind"] == "rope":
        q = st.stree_tree_rope(s["parent"], s["lengths"], s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["turns"],
                               q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS, interleaved=c["interleaved"])
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["kind"] == "attn":
        return st.stree_tree_attn(s["parent"], s["lengths"], s["q"], s["k_cache"], s["v_cache"], s["table"])
    if c["kind"] == "commit":
        lengths = st.stree_commit_kv(s["parent"], s["accepted"], s["lengths"], s["k_cache"], s["v_cache"], s["table"])
        return {"lengths": lengths, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return _pages(s, st.stree_resize_kv, st.stree_fork_kv)


# -------------------------------------------------------------------------------------------------------------- work

def work(case):
    c = case
    B, N, H, G, P, page, layers = (c[k] for k in ("batch", "nodes", "heads", "kv_heads", "headdim", "page", "layers"))
    e = 2 if c["dtype"] == "bf16" else 4
    lens = _lengths(c)
    if c["kind"] == "rope":
        # norm: square and add, then two products; rotation: three operations a value
        return {"bytes": 2 * B * N * (H + 2 * G) * P * e + B * N * 8, "flops": B * N * (H + G) * ((4 * P if c["norm"] else 0) + 3 * c["rotary"])}
    if c["kind"] == "attn":
        seen = N * (N + 1) // 2 if c["tree"] == "chain" else N * N
        return {"bytes": sum((n + N) * 2 * G * P * e for n in lens) + 2 * B * N * H * P * e,
                "flops": sum(4 * H * P * (N * n + seen) for n in lens)}
    if c["kind"] == "commit":
        # paths of such trees: a fifth to a quarter of the nodes
        return {"bytes": (B - B // 4) * max(1, N // 5) * 2 * 2 * layers * G * P * e + B * N * 4, "flops": 0}
    forks = sum(c["branches"] for n in lens if n % page)
    return {"bytes": forks * 2 * 2 * layers * G * P * page * e + 8 * B * (1 + c["branches"]) * (max(lens) // page), "flops": 0}


# ----------------------------------------------------------------------------------- the definitions in 64 bits, apart

def _paths(parent, b, nodes):
    """Per node the nodes of its path, root first (node by node on the host)."""
    if parent is None:
        return [list(range(i + 1)) for i in range(nodes)]
    paths = []
    for i, p in enumerate(parent[b].tolist()):
        paths.append((paths[p] if p >= 0 else []) + [i])
    return paths


def _exact_rope(s, c):
    N, R, P, page = c["nodes"], c["rotary"], c["headdim"], c["page"]
    out = {"q": torch.empty(s["q"].shape, dtype=torch.float64), "k_cache": s["k_cache"].cpu().double(), "v_cache": s["v_cache"].cpu().double()}
    table, turns = s["table"].cpu(), s["turns"].cpu()
    for b, n in enumerate(_lengths(c)):
        depth = [len(p) - 1 for p in _paths(s["parent"], b, N)] if s["parent"] is not None else range(N)
        pos = torch.tensor([n + d for d in depth], dtype=torch.float64)
        turn = torch.polar(torch.ones(N, R // 2, dtype=torch.float64), 2 * math.pi * torch.remainder(pos[:, None] * turns, 1.0))[:, None]
        rows = {}
        for name in "qk":
            x = s[name][b].cpu().double()
            if s[name + "_norm"] is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / P + EPS).sqrt() * s[name + "_norm"].cpu().double()
            pairs = x[..., :R].unflatten(-1, (R // 2, 2)) if c["interleaved"] else x[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
            rows[name] = torch.cat((z, x[..., R:]), -1)
        out["q"][b] = rows["q"]
        slot = torch.arange(n, n + N)
        at = table[b][slot // page].long()
        out["k_cache"][at, :, slot % page] = rows["k"]
        out["v_cache"][at, :, :, slot % page] = s["v"][b].cpu().double()
    return out


def _exact_attn(s, c):
    N, H, G, P, page = (c[k] for k in ("nodes", "heads", "kv_heads", "headdim", "page"))
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(c)):
        pages = s["table"][b, :-(-(n + N) // page)].long()
        hidden = torch.ones(N, N, dtype=torch.bool)
        for i, path in enumerate(_paths(s["parent"], b, N)):
            hidden[i, path] = False
        hidden = hidden.cuda()
        for g in range(G):
            K = s["k_cache"][pages, g].double().flatten(0, 1)[:n + N]                       # [tokens, P]
            V = s["v_cache"][pages, g].double().permute(0, 2, 1).flatten(0, 1)[:n + N]
            heads = slice(g * (H // G), (g + 1) * (H // G))
            q = s["q"][b, :, heads].double().flatten(0, 1)
            x = (q @ K.t().contiguous()) * P ** -0.5
            x.view(N, H // G, -1)[:, :, n:].masked_fill_(hidden[:, None], -math.inf)
            lse = torch.logsumexp(x, 1, keepdim=True)
            out[b, :, heads] = (torch.exp(x - lse) @ V).view(N, H // G, P)
    return out


def exact(case, seed):
    if case["kind"] in ("commit", "pages"):
        return None                                                  # rows and pages are moved, numbers counted
    s = prepare(case, seed)
    return _exact_rope(s, case) if case["kind"] == "rope" else _exact_attn(s, case)
