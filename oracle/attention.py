"""Plain forms, in 64 bits on the CPU, of the operators around the paged cache: page dealing, per-head norms with
rotation and the cache write, attention behind a shared prefix.  numpy only; values are float64 arrays."""
import numpy as np


def page_slots(kv_lens, q_lens, page_size, free_pages, n_free, table, T, pos_base=0):
    """-> (kv_lens after, q_offsets, positions, slots, info, table after)"""
    table = np.array(table, np.int64)
    B, width = table.shape
    n_free = max(0, min(int(n_free), len(free_pages)))
    after, offs, taken, asked, refused = [], [0], 0, 0, 0
    pos, slots = [], []
    for b in range(B):
        kv, q = max(int(kv_lens[b]), 0), max(int(q_lens[b]), 0)
        have, want = -(-kv // page_size), -(-(kv + q) // page_size)
        ok = want <= width
        if ok:
            first = asked
            asked += want - have
            ok = want == have or asked <= n_free
        if ok:
            for j in range(have, want):
                table[b, j] = free_pages[n_free - 1 - (first + j - have)]
            taken += want - have
        refused += not ok
        after.append(kv + q if ok else kv)
        offs.append(offs[-1] + q)
        for p in range(kv, kv + q):
            pos.append(pos_base + p)
            page = table[b, p // page_size] if ok else -1
            slots.append(page * page_size + p % page_size if 0 <= page < 2 ** 31 // page_size else -1)  # -1 too for a page that no cache can have
    pad = max(0, T - len(pos))
    return (np.array(after), np.array(offs), np.array(pos + [-1] * pad)[:T], np.array(slots + [-1] * pad)[:T],
            np.array([n_free - taken, taken, refused, offs[-1]]), table)


def rope_angles(base, rot, n_pos):
    a = np.arange(n_pos, dtype=np.float64)[:, None] * base ** (-2.0 * np.arange(rot // 2) / rot)
    return np.concatenate([np.cos(a), np.sin(a)], 1)


def head_rope(x, gamma, eps, cos_sin, positions, sections, rot, pairs):
    """x [T, H, D]; positions [axes, T] -> (y, size of what each result was made of)"""
    z = x.copy()
    if gamma is not None:
        z = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gamma
    y, size = z.copy(), np.abs(z)
    i = 0
    for a, n in enumerate(sections):
        for _ in range(n):
            c, s = cos_sin[positions[a], i][:, None], cos_sin[positions[a], rot // 2 + i][:, None]
            u, w = (2 * i, 2 * i + 1) if pairs else (i, i + rot // 2)
            y[:, :, u], y[:, :, w] = z[:, :, u] * c - z[:, :, w] * s, z[:, :, w] * c + z[:, :, u] * s
            size[:, :, u] = size[:, :, w] = np.hypot(z[:, :, u], z[:, :, w])
            i += 1
    return y, size


def prefix_attention(q, K, V, prefix_pages, prefix_len, table, kv_lens, q_offsets, scale, rows=None):
    """q [T, Hq, D]; K, V [pages, Hkv, ps, D] -> (o [T, Hq, D], lse [T, Hq], average of |v| under the weights, largest sum of |q k|);
    `rows`: only these, others are left at zeros and -infinity"""
    T, Hq, D = q.shape
    Hkv, ps = K.shape[1], K.shape[2]
    G = Hq // Hkv
    o, av, lse, big = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    wanted = np.ones(T, bool) if rows is None else np.isin(np.arange(T), rows)

    def tokens(C, pages, n):
        j = np.arange(n)
        return C[np.asarray(pages, np.int64)[j // ps], :, j % ps]
    for b in range(len(kv_lens)):
        t0, t1 = int(q_offsets[b]), int(q_offsets[b + 1])
        L = max(int(kv_lens[b]), 0)
        if not wanted[t0:t1].any():
            continue
        k, v = (np.concatenate([tokens(C, pg, n) for pg, n in ((prefix_pages, prefix_len), (table[b], L)) if n] or [np.zeros((0, Hkv, D))])
                for C in (K, V))
        for t in np.flatnonzero(wanted[t0:t1]) + t0:
            n = prefix_len + max(0, L - (t1 - t0) + (t - t0) + 1)
            if n == 0:
                continue
            for h in range(Hq):
                kk, vv = k[:n, h // G], v[:n, h // G]
                s = scale * (kk @ q[t, h])
                top = s.max()
                w = np.exp(s - top)
                den = w.sum()
                o[t, h], av[t, h], lse[t, h] = w @ vv / den, w @ np.abs(vv) / den, top + np.log(den)
                big[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max()
    return o, lse, av, big
