"""Plain fp64 forms of the attention layers' operators over a paged cache, for the tests: written from the definitions,
sequence by sequence and entry by entry.  Caches, tables and pools are numpy arrays and are changed in place.

``k`` [pages, heads, page, P], ``v`` [pages, heads, P, page]; token t of a sequence is row t % page of page
table[b, t // page].  Status codes as in include/stree.h."""
from __future__ import annotations

import numpy as np

ACCEPTED, LENGTH, PAGE, POOL, HELD = -1, -2, -3, -4, -5


def paths(parent, n):
    """Per node the nodes of its path, root first; (None, first bad node + 1) for a bad tree."""
    if parent is None:
        return [list(range(i + 1)) for i in range(n)], 0
    out = []
    for i in range(n):
        p = int(parent[i])
        if (p != -1) if i == 0 else not 0 <= p < i:
            return None, i + 1
        out.append((out[p] if i else []) + [i])
    return out, 0


def _check(parent, b, length, n, table, page):
    if length + n > table.shape[1] * page:
        return None, LENGTH
    return paths(None if parent is None else parent[b], n)


def _pages_ok(table, b, first, last, page, npages):
    return all(0 <= table[b, j] < npages for j in range(first // page, (last - 1) // page + 1))


def rope(parent, lengths, q, k, v, k_cache, v_cache, table, turns, q_norm, k_norm, eps, interleaved, scale):
    """-> (q_out, status, and per value of q and k the |u| + |w| that its rounding errors are relative to)."""
    B, N, H, P = q.shape
    npages, _, page, _ = k_cache.shape
    out, size_q, size_k = np.zeros(q.shape), np.zeros(q.shape), np.zeros(k.shape)
    status = np.zeros(B, np.int32)
    R = 2 * len(turns)
    for b in range(B):
        n = int(lengths[b])
        if n < 0:
            continue
        path, bad = _check(parent, b, n, N, table, page)
        if not bad and not _pages_ok(table, b, n, n + N, page, npages):
            bad = PAGE
        status[b] = bad
        if bad:
            continue
        for i in range(N):
            pos = n + len(path[i]) - 1
            t = turns * pos
            a = 2 * np.pi * (t - np.floor(t))
            rows = []
            for x, w in ((q[b, i], q_norm), (k[b, i], k_norm)):
                x = x.astype(np.float64)
                if w is not None:
                    x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
                first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
                y, m = x.copy(), np.abs(x)
                y[:, first] = scale * (x[:, first] * np.cos(a) - x[:, second] * np.sin(a))
                y[:, second] = scale * (x[:, first] * np.sin(a) + x[:, second] * np.cos(a))
                m[:, first] = m[:, second] = scale * (np.abs(x[:, first]) + np.abs(x[:, second]))
                rows.append((y, m))
            (out[b, i], size_q[b, i]), (key, size_k[b, i]) = rows
            pg, at = table[b, (n + i) // page], (n + i) % page
            k_cache[pg, :, at] = key
            v_cache[pg, :, :, at] = v[b, i]
    return out, status, size_q, size_k


def gather(k_cache, v_cache, table, b, tokens):
    """Rows of the first tokens of a sequence: keys and values [tokens, heads, P]."""
    page = k_cache.shape[2]
    t = np.arange(tokens)
    pg = table[b, t // page]
    return k_cache[pg, :, t % page], v_cache[pg, :, :, t % page]


def attn(parent, lengths, q, k_cache, v_cache, table, scale):
    """-> (out, status, sum of p |V| per value, largest scale * sum |q| |k| per row): what rounding errors are relative to."""
    B, N, H, P = q.shape
    npages, G, page, _ = k_cache.shape
    out, weight, score = np.zeros(q.shape), np.zeros(q.shape), np.zeros((B, N, H))
    status = np.zeros(B, np.int32)
    for b in range(B):
        n = int(lengths[b])
        if n < 0:
            continue
        path, bad = _check(parent, b, n, N, table, page)
        if not bad and not _pages_ok(table, b, 0, n + N, page, npages):
            bad = PAGE
        status[b] = bad
        if bad:
            continue
        K, V = gather(k_cache, v_cache, table, b, n + N)
        K, V = K.astype(np.float64), V.astype(np.float64)
        for i in range(N):
            seen = list(range(n)) + [n + j for j in path[i]]
            for h in range(H):
                g = h // (H // G)
                Ks, Vs, x = K[seen, g], V[seen, g], q[b, i, h].astype(np.float64)
                s = scale * (Ks @ x)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, i, h] = p @ Vs
                weight[b, i, h] = p @ np.abs(Vs)
                score[b, i, h] = abs(scale) * (np.abs(Ks) @ np.abs(x)).max()
    return out, status, weight, score


def commit(parent, accepted, lengths, n, k_cache, v_cache, table):
    """Caches [layers, pages, ...]; -> (new lengths, status)."""
    npages, page = k_cache.shape[1], k_cache.shape[3]
    out, status = np.array(lengths, np.int32), np.zeros(len(lengths), np.int32)
    for b in range(len(lengths)):
        at, k = int(lengths[b]), int(accepted[b])
        if at < 0:
            continue
        path, bad = _check(parent, b, at, n, table, page)
        if not bad and not -1 <= k < n:
            bad = ACCEPTED
        if not bad and k >= 0 and not _pages_ok(table, b, at, at + k + 1, page, npages):
            bad = PAGE
        status[b] = bad
        if bad or k < 0:
            continue
        place = lambda t: (table[b, t // page], t % page)  # noqa: E731
        rows = [(k_cache[:, place(at + j)[0], :, place(at + j)[1]].copy(), v_cache[:, place(at + j)[0], :, :, place(at + j)[1]].copy())
                for j in path[k]]
        for t, (kr, vr) in enumerate(rows):
            pg, r = place(at + t)
            k_cache[:, pg, :, r] = kr
            v_cache[:, pg, :, :, r] = vr
        out[b] = at + len(rows)
    return out, status


def resize(tokens, held, table, refs, free, nfree, page):
    """-> status."""
    B, M = table.shape
    npages, status = len(refs), np.zeros(len(tokens), np.int32)
    if not 0 <= nfree[0] <= npages:
        return np.full(B, POOL, np.int32)
    need = np.array(held, np.int64)
    for b in range(B):
        if not 0 <= held[b] <= M or tokens[b] > M * page:
            status[b] = LENGTH
        elif tokens[b] >= 0:
            need[b] = -(-int(tokens[b]) // page)
    dropped = [(b, j) for b in range(B) for j in range(max(need[b], 0), max(held[b], 0)) if need[b] < held[b]]
    count = {}
    for b, j in dropped:
        count[int(table[b, j])] = count.get(int(table[b, j]), 0) + 1
    for b, j in dropped:
        pg = int(table[b, j])
        if not 0 <= pg < npages:
            status[b] = PAGE
        elif count[pg] > refs[pg]:
            status[b] = PAGE
        table[b, j] = -1
    done = set()
    order = []
    for pg in (p for p in count):                        # (insertion order: the order of the first entries)
        if 0 <= pg < npages and pg not in done:
            done.add(pg)
            left = refs[pg] - count[pg]
            if left == 0:
                order.append(pg)
            refs[pg] = max(left, 0)
    for pg in order:
        free[nfree[0]] = pg
        nfree[0] += 1
    stuck = False
    for b in range(B):
        more = need[b] - held[b]
        if status[b] == LENGTH:
            continue
        if more > 0 and (stuck or more > nfree[0]):
            stuck, status[b] = True, POOL
            continue
        for j in range(held[b], need[b]):
            nfree[0] -= 1
            pg = free[nfree[0]]
            table[b, j] = pg
            if 0 <= pg < npages:
                refs[pg] = 1
            else:
                status[b] = PAGE
        held[b] = need[b]
    return status


def fork(src, dst, lengths, held, table, refs, free, nfree, k_cache, v_cache):
    """Caches [layers, pages, ...]; -> status per fork."""
    B, M = table.shape
    npages, page = len(refs), k_cache.shape[3]
    status = np.zeros(len(src), np.int32)
    if not 0 <= nfree[0] <= npages:
        return np.full(len(src), POOL, np.int32)
    was_len, was_held, was_refs, taken, missing = np.array(lengths), np.array(held), np.array(refs), set(), False
    for f in range(len(src)):
        s, d = int(src[f]), int(dst[f])
        if not (0 <= s < B and 0 <= d < B) or was_len[s] < 0 or not 0 <= was_held[s] <= M or -(-was_len[s] // page) > was_held[s]:
            status[f] = LENGTH
            continue
        pages = [int(p) for p in table[s, :-(-was_len[s] // page)]]
        if any(not 0 <= p < npages or was_refs[p] <= 0 for p in pages):
            status[f] = PAGE
            continue
        if was_held[d] != 0 or d in taken:
            status[f] = HELD
            continue
        taken.add(d)
        full, rest = was_len[s] // page, was_len[s] % page
        if rest:
            missing = missing or nfree[0] == 0
            if missing:
                status[f] = POOL
                continue
            nfree[0] -= 1
            pg = free[nfree[0]]
            if not 0 <= pg < npages:
                status[f] = PAGE
                continue
            table[d, full] = pg
            refs[pg] = 1
            k_cache[:, pg] = k_cache[:, pages[full]]
            v_cache[:, pg] = v_cache[:, pages[full]]
        for j in range(full):
            table[d, j] = pages[j]
            refs[pages[j]] += 1
        held[d], lengths[d] = full + (rest > 0), was_len[s]
    return status
