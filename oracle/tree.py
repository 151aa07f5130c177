"""Plain forms, in 64 bits on the CPU, of the operators of speculative decoding over the paged cache: bits and positions of trees of
drafted tokens, attention of their rows, the accepted path, keys and values moved between slots, forked and freed pages, log
probabilities.  numpy only; one thing after the other."""
import numpy as np


def tree_mask(parents, q_offsets, kv_lens, T, words, pos_base=0):
    """-> (mask uint64 [T, words], positions [T])"""
    mask, pos = np.zeros((T, words), np.uint64), np.full(T, -1)
    for b, L in enumerate(kv_lens):
        t, n = int(q_offsets[b]), int(q_offsets[b + 1] - q_offsets[b])
        for i in range(n):
            depth = i
            if n <= 64 * words:
                at, depth = i, -1
                while True:
                    mask[t + i, at // 64] |= np.uint64(1 << (at % 64))
                    depth += 1
                    if not 0 <= parents[t + at] < at:
                        break
                    at = int(parents[t + at])
            pos[t + i] = max(pos_base + max(int(L), 0) - n + depth, -1)
    return mask, pos


def tree_attention(q, K, V, prefix_pages, prefix_len, table, kv_lens, q_offsets, mask, scale):
    """q [T, Hq, D]; K, V [pages, Hkv, ps, D]; mask uint64 [T, words] -> (o, lse, average of |v| under the weights, largest sum of |q k|)"""
    T, Hq, D = q.shape
    Hkv, ps = K.shape[1], K.shape[2]
    G, words = Hq // Hkv, mask.shape[1]
    o, av, lse, big = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf), np.zeros((T, Hq))

    def tokens(C, pages, n):
        j = np.arange(n)
        return C[np.asarray(pages, np.int64)[j // ps], :, j % ps]
    for b in range(len(kv_lens)):
        t0, t1 = int(q_offsets[b]), int(q_offsets[b + 1])
        n, L = t1 - t0, max(int(kv_lens[b]), 0)
        if n == 0:
            continue
        k, v = (np.concatenate([tokens(C, pg, m) for pg, m in ((prefix_pages, prefix_len), (table[b], L)) if m] or [np.zeros((0, Hkv, D))])
                for C in (K, V))
        for i in range(n):
            new = np.arange(L) - (L - n)  # which of the new tokens a cached one is
            sees = new <= i
            if n <= 64 * words:
                bits = np.array([(int(mask[t0 + i, x // 64]) >> (x % 64)) & 1 if 0 <= x < n else 0 for x in range(n)], bool)
                sees &= (new < 0) | bits[np.clip(new, 0, n - 1)]
            sees = np.concatenate([np.ones(prefix_len, bool), sees])
            if not sees.any():
                continue
            for h in range(Hq):
                kk, vv = k[sees, h // G], v[sees, h // G]
                s = scale * (kk @ q[t0 + i, h])
                top = s.max()
                w = np.exp(s - top)
                den = w.sum()
                o[t0 + i, h], av[t0 + i, h], lse[t0 + i, h] = w @ vv / den, w @ np.abs(vv) / den, top + np.log(den)
                big[t0 + i, h] = (np.abs(kk) @ np.abs(q[t0 + i, h])).max()
    return o, lse, av, big


def tree_accept(parents, tokens, choices, q_offsets, kv_lens, slots, T):
    """-> (path [T], n_accepted [B], next_tokens [B], kv_lens after [B], src_slots [T])"""
    path, src = np.full(T, -1), np.full(T, -1)
    count, following, lens = [], [], []
    for b, L in enumerate(kv_lens):
        t, n = int(q_offsets[b]), int(q_offsets[b + 1] - q_offsets[b])
        if n == 0 or slots[t] < 0:
            count.append(0), following.append(-1), lens.append(int(L))
            continue
        line = [0]
        while True:
            nxt = [i for i in range(line[-1] + 1, n) if parents[t + i] == line[-1] and (tokens[t + i] < 0 or tokens[t + i] == choices[t + line[-1]])]
            if not nxt:
                break
            line.append(nxt[0])
        path[t:t + len(line)] = line
        src[t:t + len(line)] = [slots[t + i] for i in line]
        count.append(len(line)), following.append(int(choices[t + line[-1]])), lens.append(int(L) - n + len(line))
    return path, np.array(count, int), np.array(following, int), np.array(lens, int), src


def cache_move(C, src, dst, offsets):
    """C [layers, pages, Hkv, ps, D], changed in place, a pair after the other"""
    ps, slots = C.shape[3], C.shape[1] * C.shape[3]
    for g in range(len(offsets) - 1):
        for i in range(offsets[g], offsets[g + 1]):
            a, b = int(src[i]), int(dst[i])
            if 0 <= a < slots and 0 <= b < slots:
                C[:, b // ps, :, b % ps] = C[:, a // ps, :, a % ps]


def page_fork(src, dst, kv_lens, table, refs, free_pages, n_free, ps):
    """-> (kv_lens, table, refs, src_slots [N, ps], dst_slots, info)"""
    kv, table, refs = [int(x) for x in kv_lens], np.array(table, np.int64), np.array(refs, np.int64)
    B, width = table.shape
    n_free = max(0, min(int(n_free), len(free_pages)))
    out = [np.full((len(src), ps), -1) for _ in range(2)]
    asked = taken = refused = shared = 0
    for f, (a, b) in enumerate(zip(src, dst)):
        ok = 0 <= a < B and 0 <= b < B and b not in list(src) and b not in list(dst[:f]) and kv[a] <= width * ps
        L = max(kv[a], 0) if ok else 0
        full, part = divmod(L, ps)
        if ok and part:
            asked += 1
            ok = asked <= n_free
        if not ok:
            refused += 1
            continue
        for j in range(full):
            page = table[b, j] = table[a, j]
            shared += 1
            if 0 <= page < len(refs):
                refs[page] += 1
        if part:
            taken += 1
            was, page = table[a, full], free_pages[n_free - asked]
            table[b, full] = page
            if 0 <= was < len(refs) and 0 <= page < len(refs):
                out[0][f, :part], out[1][f, :part] = was * ps + np.arange(part), page * ps + np.arange(part)
        kv[b] = L
    return np.array(kv, int), table, refs, out[0], out[1], np.array([n_free - taken, taken, refused, shared])


def page_free(kv_lens, new_lens, table, refs, free_pages, n_free, ps, n_pages):
    """-> (refs, free_pages, info)"""
    refs = None if refs is None else np.array(refs, np.int64)
    free = np.array(free_pages, np.int64)
    n_free = max(0, min(int(n_free), len(free)))
    dead, kept, ignored = set(), 0, 0
    for b in range(len(kv_lens)):
        new = 0 if new_lens is None else max(int(new_lens[b]), 0)
        for j in range(-(-new // ps), min(-(-max(int(kv_lens[b]), 0) // ps), table.shape[1])):
            page = int(table[b, j])
            if not 0 <= page < n_pages or page in dead:
                ignored += 1
            elif refs is not None and refs[page] > 0:
                refs[page] -= 1
                kept += 1
            else:
                dead.add(page)
    room = [p for p in sorted(dead)][:len(free) - n_free]
    free[n_free:n_free + len(room)] = room
    if refs is not None:
        refs[list(dead)] = 0
    return refs, free, np.array([n_free + len(room), len(room), kept, ignored + len(dead) - len(room)])


def token_logprobs(x, tokens, k, scale):
    """x [T, V]; tokens [T, n] -> (log probabilities [T, n], ids [T, k], their log probabilities, lse [T], entropy [T])"""
    T, V = x.shape
    lp, ids, top = np.zeros(tokens.shape), np.full((T, k), -1), np.full((T, k), np.nan)
    lse, entropy = np.full(T, np.nan), np.full(T, np.nan)
    for t in range(T):
        given = [(i, j) for i, j in enumerate(tokens[t]) if 0 <= j < V]
        if np.isnan(x[t]).any() or np.isposinf(x[t]).any():
            for i, _ in given:
                lp[t, i] = np.nan
            continue
        order = np.argsort(-x[t], kind="stable")[:k]
        ids[t] = order
        if np.isneginf(x[t]).all():
            p, lse[t], entropy[t] = np.full(V, -np.inf), -np.inf, 0
        else:
            z = scale * x[t]
            size = np.log(np.exp(z - z.max()).sum())
            lse[t], p = z.max() + size, z - z.max() - size  # by differences: a row of the type's lowest value is even
            some = ~np.isneginf(p)
            entropy[t] = -(np.exp(p[some]) * p[some]).sum()
        top[t] = p[order]
        for i, j in given:
            lp[t, i] = p[j]
    return lp, ids, top, lse, entropy
