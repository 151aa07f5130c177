"""The operators of speculative decoding over a paged cache: drafted tokens form a tree, one step scores the whole tree, and what
the model agrees with stays in the cache.

kind    one pass
tree    which drafted tokens a row sees and its position from the tree's parents, then attention of the tree's rows over a shared
        prefix, the request's own tokens and the row's ancestors
logp    log probabilities of given tokens, the entropy and the top alternatives of rows of logits
commit  the accepted path of every tree, its keys and values moved behind the request's tokens in all layers, the pages behind it freed
fork    one step of a search over continuations: pages of the dropped rows freed, kept rows forked into them, the part of a page that
        each fork writes next copied in all layers

Head layouts are those of the benchmark configurations (32 query heads on 8 or 4 key/value heads of 128 channels) and a generic
one with heads of 64; vocabularies and lengths are generic, odd ones among them.
"""
import math
import random

import torch

own = False
DEV = "cuda"


def listed():
    return [
        # one request, a few drafted tokens: latency
        dict(name="tree_1x8", kind="tree", B=1, n=8, chunk=0, prefix=0, kv=700, Hq=32, Hkv=8, D=128, ps=16, words=1, lens=1),
        # an ordinary batch with contexts of its own, trees of up to 16 tokens
        dict(name="tree_24x16", kind="tree", B=24, n=16, chunk=0, prefix=0, kv=3100, Hq=32, Hkv=8, D=128, ps=64, words=1, lens=2),
        # a batch behind a system prompt, larger trees, chunks of new prompts in the same step
        dict(name="tree_48x32_prefix", kind="tree", B=48, n=32, chunk=190, prefix=4096, kv=700, Hq=32, Hkv=4, D=128, ps=32, words=1, lens=3),
        # few requests with long contexts, the widest trees of one word and more, small heads
        dict(name="tree_6x97_long", kind="tree", B=6, n=97, chunk=0, prefix=0, kv=24000, Hq=24, Hkv=8, D=64, ps=128, words=2, lens=4),
        # one row of logits after a decode step of one request
        dict(name="logp_1", kind="logp", T=1, V=131072, dtype="bf16", tokens=1, top=8, scale=1.0),
        # a decode batch, single precision logits of an odd vocabulary, tempered
        dict(name="logp_100", kind="logp", T=100, V=50001, dtype="f32", tokens=1, top=20, scale=1.25),
        # a tree's candidate tokens for every row, no alternatives
        dict(name="logp_511_six", kind="logp", T=511, V=32000, dtype="bf16", tokens=6, top=0, scale=1.0),
        # the log probabilities of a long prompt
        dict(name="logp_2048", kind="logp", T=2048, V=131072, dtype="bf16", tokens=1, top=5, scale=1.0),
        # a small batch, one layer
        dict(name="commit_4", kind="commit", B=4, n=8, kv=200, layers=1, Hkv=8, D=128, ps=16, lens=5),
        # a large batch, all layers of a cache in one call
        dict(name="commit_200", kind="commit", B=200, n=24, kv=250, layers=4, Hkv=8, D=128, ps=32, lens=6),
        # a small search: four rows go on from two others
        dict(name="fork_4", kind="fork", N=4, B=16, kv=300, layers=1, Hkv=8, D=128, ps=16, lens=7),
        # many rows dropped and forked at once, large pages
        dict(name="fork_150", kind="fork", N=150, B=512, kv=300, layers=4, Hkv=4, D=128, ps=64, lens=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "logp", "logp", "commit", "fork"])
    ps = rng.choice([16, 32, 64, 128])
    lens = rng.randrange(100, 10 ** 6)
    if kind == "logp":
        V = rng.choice([_log_int(rng, 1000, 131072), 32000, 50257, 128256])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(kind=kind, T=max(1, min(_log_int(rng, 1, 4000), (200 if dtype == "bf16" else 100) * 10 ** 6 // V)), V=V, dtype=dtype,
                    tokens=rng.choice([0, 1, 1, 1, 2, 9]), top=rng.choice([0, 1, 5, 8, 20, 33]), scale=rng.choice([1.0, 1.0, 0.7, 1.6]))
    Hq, Hkv, D = rng.choice([(32, 8, 128), (32, 4, 128), (24, 8, 64), (12, 12, 64), (40, 8, 128), (28, 4, 128)])
    if kind == "tree":
        B = _log_int(rng, 1, 100)
        words = rng.choice([1, 1, 1, 2, 4])
        n = min(_log_int(rng, 2, 64 * words), max(2, 1600 // B))
        prefix = rng.choice([0, 0, _log_int(rng, 16, 4000)])
        return dict(kind=kind, B=B, n=n, chunk=rng.choice([0, 0, 0, 64 * words + _log_int(rng, 1, 200)]) if B <= 40 else 0, prefix=prefix, kv=min(_log_int(rng, 4, 24000), 140000 // B),
                    Hq=Hq, Hkv=Hkv, D=D, ps=ps, words=words, lens=lens)
    layers = rng.choice([1, 1, 2, 4])
    if kind == "commit":
        return dict(kind=kind, B=_log_int(rng, 1, 200), n=_log_int(rng, 2, 64), kv=_log_int(rng, 1, 250), layers=layers, Hkv=Hkv, D=D, ps=ps, lens=lens)
    B = _log_int(rng, 2, 500)
    return dict(kind=kind, N=max(1, min(B // 2, _log_int(rng, 1, 150))), B=B, kv=_log_int(rng, 1, 300), layers=layers, Hkv=min(Hkv, 8), D=D, ps=ps, lens=lens)


# ---- lengths: the case's own, so that every seed has the same work; a seed deals them to the requests ----


def _lengths(case):
    """(tokens a request has cached before the step, tokens of the step), one pair a request"""
    rng = random.Random(case["lens"])
    out = []
    for b in range(case["B"]):
        kv = rng.randint(case["kv"] // 4, case["kv"]) if b % 8 else case["kv"]
        n = rng.randint(case["n"] // 2 + 1, case["n"]) if b % 5 else case["n"]
        if case.get("chunk") and b % 16 == 5:
            n = case["chunk"]
        out.append((kv, n))
    return out


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *size, std=1.0, dtype=torch.bfloat16):
    """made in pieces: a long cache is large"""
    out = torch.empty(size, dtype=dtype, device=DEV)
    flat = out.view(-1)
    step = 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device=DEV) * std
    return out


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _rows(offs):
    """request and place inside it of every row"""
    offs = torch.tensor(offs, device=DEV)
    req = torch.repeat_interleave(torch.arange(offs.numel() - 1, device=DEV), offs[1:] - offs[:-1])
    return req, torch.arange(req.numel(), device=DEV) - offs[req]


def _parents(g, place):
    """half of the tokens continue the one before them, the others any earlier one; a request's first token is the root"""
    u = torch.rand(2, place.numel(), generator=g, device=DEV, dtype=torch.float64)
    return torch.where(u[0] < 0.5, place - 1, (u[1] * place).long().clamp(max=place - 1)).int()


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["kind"] == "logp":
        T, V = case["T"], case["V"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["logits"] = _randn(g, T, V, std=3.0, dtype=dtype)
        peaks = torch.randint(0, V // 6, (T, 6), generator=g, device=DEV) + torch.arange(6, device=DEV) * (V // 6)  # a model is sure of a few tokens
        s["logits"].scatter_(1, peaks, (8 + 6 * torch.rand(T, 6, generator=g, device=DEV)).to(dtype))
        s["given"] = torch.cat([peaks[:, :1], torch.randint(0, V, (T, max(case["tokens"], 1)), generator=g, device=DEV)], 1)[:, :case["tokens"]].int().contiguous()
        if own:
            import paper_2604_12782_amd as osc
            s["workspace"] = torch.empty(osc.osc_token_logprobs_workspace_bytes(T, V, case["top"]), dtype=torch.uint8, device=DEV)
        return s
    ps, D, Hkv, B = case["ps"], case["D"], case["Hkv"], case["B"]
    rng = random.Random(seed * 7919 + 1)
    if case["kind"] == "fork":
        N, layers = case["N"], case["layers"]
        lens = random.Random(case["lens"])
        kv = [lens.randint(1, case["kv"]) for _ in range(B)]
        rng.shuffle(kv)
        rows = rng.sample(range(B), B)
        dst, kept = rows[:N], rows[N:]
        src = [rng.choice(kept[:max(1, N // 2)]) for _ in range(N)]
        pages = [-(-a // ps) for a in kv]
        n_pages = sum(pages) + N + 5
        perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((B, -(-case["kv"] // ps) + 1), -1, dtype=torch.int32, device=DEV)
        table[_i32(pages)[:, None] > torch.arange(table.shape[1], device=DEV)[None]] = perm[:sum(pages)]
        new = _i32(kv)
        new[torch.tensor(dst, device=DEV)] = 0
        free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        free[:n_pages - sum(pages)] = perm[sum(pages):]
        s.update(src=_i32(src), dst=_i32(dst), kv_lens=_i32(kv), new_lens=new, table=table, refs=torch.zeros(n_pages, dtype=torch.int32, device=DEV),
                 free=free, n_free=_i32([n_pages - sum(pages)]), K=_randn(g, layers, n_pages, Hkv, ps, D), V=_randn(g, layers, n_pages, Hkv, ps, D))
        return s
    pairs = _lengths(case)
    rng.shuffle(pairs)
    kv0, n = [a for a, _ in pairs], [b for _, b in pairs]
    kv = [a + b for a, b in pairs]  # the step's tokens are in the cache by now
    offs, P = _offsets(n), case.get("prefix", 0)
    T = offs[-1]
    req, place = _rows(offs)
    parents = _parents(g, place)
    pages = [-(-a // ps) for a in kv]
    n_prefix = -(-P // ps)
    n_pages = sum(pages) + n_prefix + 2
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, max(pages)), -1, dtype=torch.int32, device=DEV)
    table[_i32(pages)[:, None] > torch.arange(table.shape[1], device=DEV)[None]] = perm[n_prefix:n_prefix + sum(pages)]
    s.update(T=T, kv_list=kv, n_list=n, offs_list=offs, parents=parents, table=table, kv_lens=_i32(kv), q_offsets=_i32(offs))
    if case["kind"] == "commit":
        layers = case["layers"]
        at = torch.tensor(kv0, device=DEV)[req] + place
        tokens = torch.randint(0, 32000, (T,), generator=g, device=DEV)
        # the model follows one of a token's continuations seven times in ten
        kept = (torch.rand(T, generator=g, device=DEV) < 0.7) & (place > 0)
        first = torch.tensor(offs, device=DEV)[req]
        child = torch.full((T + 1,), -1, device=DEV)
        child.scatter_reduce_(0, torch.where(kept, first + parents, T), torch.arange(T, device=DEV), "amax")
        choices = torch.where(child[:T] >= 0, tokens[child[:T].clamp(min=0)], torch.randint(0, 32000, (T,), generator=g, device=DEV))
        free = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        free[:2] = perm[n_pages - 2:]
        s.update(tokens=tokens.int(), choices=choices.int(), slots=(table[req, at // ps] * ps + at % ps).int(), refs=torch.zeros(n_pages, dtype=torch.int32, device=DEV),
                 free=free, n_free=_i32([2]), K=_randn(g, layers, n_pages, Hkv, ps, D), V=_randn(g, layers, n_pages, Hkv, ps, D))
        return s
    Hq = case["Hq"]
    s.update(prefix_pages=perm[:n_prefix].contiguous(), Q=_randn(g, T, Hq * D, std=1.5), K=_randn(g, n_pages, Hkv, ps, D), V=_randn(g, n_pages, Hkv, ps, D),
             scale=D ** -0.5)
    if own:
        import paper_2604_12782_amd as osc
        s["workspace"] = torch.empty(osc.osc_tree_attention_workspace_bytes(T, B, Hq, Hkv, D, P), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----


def run(s):
    return {"tree": _tree, "logp": _logp, "commit": _commit, "fork": _fork}[s["kind"]](s)


def _row_places(q_offsets, T):
    """request, place in it and number of the request's rows, from offsets on the device"""
    offs = q_offsets.long()
    t = torch.arange(T, device=DEV)
    req = torch.searchsorted(offs, t, right=True) - 1
    return req, t - offs[req], (offs[1:] - offs[:-1])[req]


def _tree_mask(parents, q_offsets, kv_lens, words, pos_base):
    """bits of a row: itself and its ancestors; position: behind the request's tokens by the number of ancestors"""
    T = parents.numel()
    req, place, n = _row_places(q_offsets, T)
    is_tree = n <= 64 * words
    sees = torch.zeros((T + 1, 64 * words), dtype=torch.bool, device=DEV)
    sees[:T] = (torch.arange(64 * words, device=DEV) == place[:, None]) & is_tree[:, None]
    first = q_offsets.long()[req]
    has = (parents >= 0) & (parents < place) & is_tree
    jump = torch.cat([torch.where(has, first + parents, T), torch.full((1,), T, device=DEV)])  # row T: nothing
    for _ in range((64 * words - 1).bit_length()):
        sees = sees | sees[jump]
        jump = jump[jump]
    sees = sees[:T]
    depth = torch.where(is_tree, sees.sum(1) - 1, place)
    bits = (sees.view(T, words, 64).long() << torch.arange(64, device=DEV)).sum(-1)
    return bits, (pos_base + kv_lens.long()[req] - n + depth).int()


def _part(q, k, v, scale, mask=None):
    """one piece of a softmax: q [..., R, D], k and v [..., L, D] -> sums over L, weights' sum, maximum"""
    a = torch.matmul(q, k.transpose(-1, -2)) * scale
    if mask is not None:
        a = a.masked_fill(~mask, -math.inf)
    m = a.amax(-1, keepdim=True)
    p = torch.exp(a - torch.where(m == -math.inf, 0, m))
    return torch.matmul(p, v), p.sum(-1, keepdim=True), m


def _join(a, b):
    m = torch.maximum(a[2], b[2])
    base = torch.where(m == -math.inf, 0, m)
    wa, wb = torch.exp(a[2] - base), torch.exp(b[2] - base)
    return a[0] * wa + b[0] * wb, a[1] * wa + b[1] * wb, m


def _cached(C, pages, n):
    """rows 0..n-1 of every request (or of the prefix) from its pages: [..., Hkv, n, D] in 32 bits"""
    x = C[pages].float()  # [..., pages, Hkv, ps, D]
    return x.transpose(-4, -3).flatten(-3, -2)[..., :n, :]


def _tree(s):
    T, Hq, Hkv, D, P, words, B, scale = s["T"], s["Hq"], s["Hkv"], s["D"], s["prefix"], s["words"], s["B"], s["scale"]
    if own:
        import paper_2604_12782_amd as osc
        mask, pos = osc.osc_tree_mask(s["parents"], s["q_offsets"], s["kv_lens"], words, P)
        o, lse = osc.osc_tree_attention(s["Q"], Hq, Hkv, D, s["K"], s["V"], s["prefix_pages"], P, s["table"], s["kv_lens"], s["q_offsets"], mask, scale,
                                        want_lse=True, workspace=s["workspace"])
        return mask, pos, o, lse
    bits, pos = _tree_mask(s["parents"], s["q_offsets"], s["kv_lens"], words, P)
    G, most, longest = Hq // Hkv, max(s["n_list"]), max(s["kv_list"])
    req, place, n = _row_places(s["q_offsets"], T)
    j = torch.arange(longest, device=DEV) - (s["kv_lens"].long()[req] - n)[:, None]  # the step's token that a cached one is, or below 0
    word = bits.gather(1, (j >> 6).clamp(0, words - 1))
    sees = (j < 0) | ((j <= place[:, None]) & ((n > 64 * words)[:, None] | ((word >> (j & 63)) & 1).bool()))
    q = torch.zeros((B, most, Hkv, G, D), device=DEV)
    q[req, place] = s["Q"].float().view(T, Hkv, G, D)
    full = torch.ones((B, most, longest), dtype=torch.bool, device=DEV)
    full[req, place] = sees
    pages = s["table"].long().clamp(min=0)
    k, v = _cached(s["K"], pages, longest), _cached(s["V"], pages, longest)  # [B, Hkv, L, D]
    rows = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, most * G, D)
    acc = _part(rows, k, v, scale, full.repeat_interleave(G, 1)[:, None])
    acc = [x.view(B, Hkv, most, G, -1)[req, :, place] for x in acc]  # [T, Hkv, G, .]
    if P:
        pages = s["prefix_pages"].long()
        k, v = _cached(s["K"], pages, P), _cached(s["V"], pages, P)
        rows = s["Q"].float().view(T, Hkv, G, D).transpose(0, 1).reshape(Hkv, T * G, D)
        acc = _join(acc, [x.view(Hkv, T, G, -1).transpose(0, 1) for x in _part(rows, k, v, scale)])
    num, den, top = acc
    return bits, pos, (num / den).reshape(T, Hq * D).bfloat16(), (top + torch.log(den)).reshape(T, Hq)


def _logp(s):
    top, scale, given = s["top"], s["scale"], s["given"]
    if own:
        import paper_2604_12782_amd as osc
        return osc.osc_token_logprobs(s["logits"], given if s["tokens"] else None, top, scale, workspace=s["workspace"])
    raw = s["logits"].float()
    x = raw * scale
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(1, keepdim=True)
    lse = m + torch.log(z)
    entropy = torch.log(z) - (e * (x - m)).sum(1, keepdim=True) / z
    ids = best = None
    if top:
        b = (raw + 0.0).view(torch.int32)  # in the order of the values; equal ones by their place
        key = (b ^ ((b >> 31) & 0x7fffffff)).long() * (1 << 32) + (0xffffffff - torch.arange(s["V"], device=DEV))
        ids = 0xffffffff - (torch.topk(key, top, dim=1).values & 0xffffffff)
        best = x.gather(1, ids) - lse
        ids = ids.int()
    return (x.gather(1, given.long()) - lse if s["tokens"] else None), ids, best, lse[:, 0], entropy[:, 0]


def _moved(C, src, dst, ps):
    """tokens of slots `src` written to slots `dst` in all layers"""
    C[:, dst // ps, :, dst % ps] = C[:, src // ps, :, src % ps]


def _free(old, new, table, refs, free, n_free, ps):
    """pages behind the new lengths lose a holder; those without any go to the list in the order of their numbers"""
    at = torch.arange(table.shape[1], device=DEV)[None]
    gone = (at >= ((new.clamp(min=0) + ps - 1) // ps)[:, None]) & (at < ((old + ps - 1) // ps)[:, None])
    count = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=DEV)
    count.index_add_(0, torch.where(gone, table, refs.numel()).view(-1), torch.ones(table.numel(), dtype=torch.int32, device=DEV))
    count = count[:-1]
    freed = (count > 0) & (count > refs)
    kept = torch.minimum(count, refs).sum()
    refs.copy_((refs - count).clamp(min=0))
    place = n_free[0] + freed.cumsum(0) - 1
    ids = torch.arange(refs.numel(), device=DEV)
    m = freed.sum()
    wide = torch.cat([free, free[:1]])
    wide[torch.where(freed, place, free.numel())] = ids.int()
    free.copy_(wide[:-1])
    return torch.stack([n_free[0] + m, m, kept, m - m]).int()


def _commit(s):
    ps, T = s["ps"], s["T"]
    if own:
        import paper_2604_12782_amd as osc
        path, count, following, lens, src = osc.osc_tree_accept(s["parents"], s["tokens"], s["choices"], s["q_offsets"], s["kv_lens"], s["slots"])
        osc.osc_cache_move(s["K"], s["V"], src, s["slots"], s["q_offsets"])
        info = osc.osc_page_free(s["kv_lens"], lens, s["table"], s["free"], s["n_free"], ps, s["refs"])
        return path, count, following, lens, src, s["K"], s["V"], s["refs"], s["free"], info
    req, place, n = _row_places(s["q_offsets"], T)
    first = s["q_offsets"].long()[req]
    up = torch.where((s["parents"] >= 0) & (s["parents"] < place), first + s["parents"], T)
    t = torch.arange(T, device=DEV)
    agreed = torch.cat([s["choices"], s["choices"][:1]])[up] == s["tokens"]
    lowest = torch.full((T + 1,), T, device=DEV).scatter_reduce_(0, torch.where(agreed, up, T), t, "amin")
    good = torch.cat([(place == 0) | (agreed & (up < T) & (lowest[up] == t)), torch.ones(1, dtype=torch.bool, device=DEV)])
    jump = torch.cat([torch.where(place == 0, T, up), torch.full((1,), T, device=DEV)])
    for _ in range((s["n"] - 1).bit_length()):
        good = good & good[jump]
        jump = jump[jump]
    good = good[:T]
    before = torch.cat([good.new_zeros(1, dtype=torch.long), good.long().cumsum(0)])
    offs = s["q_offsets"].long()
    count = before[offs[1:]] - before[offs[:-1]]
    path = torch.full((T + 1,), -1, device=DEV)
    path[torch.where(good, first + before[:T] - before[first], T)] = place
    path = path[:T]
    src = torch.where(path >= 0, s["slots"].long()[(first + path).clamp(min=0)], -1)
    following = s["choices"][offs[:-1] + path[(offs[:-1] + count - 1)]]
    lens = (s["kv_lens"] - (offs[1:] - offs[:-1]) + count).int()
    move = src >= 0
    for C in (s["K"], s["V"]):
        _moved(C, src[move], s["slots"].long()[move], ps)
    info = _free(s["kv_lens"], lens, s["table"], s["refs"], s["free"], s["n_free"], ps)
    return path.int(), count.int(), following, lens, src.int(), s["K"], s["V"], s["refs"], s["free"], info


def _fork(s):
    ps, N = s["ps"], s["N"]
    if own:
        import paper_2604_12782_amd as osc
        freed = osc.osc_page_free(s["kv_lens"], s["new_lens"], s["table"], s["free"], s["n_free"], ps, s["refs"])
        src, dst, info = osc.osc_page_fork(s["src"], s["dst"], s["kv_lens"], s["table"], s["refs"], s["free"], freed[:1], ps)
        osc.osc_cache_move(s["K"], s["V"], src, dst)
        return s["kv_lens"], s["table"], s["refs"], s["free"], freed, src, dst, info, s["K"], s["V"]
    freed = _free(s["kv_lens"], s["new_lens"], s["table"], s["refs"], s["free"], s["n_free"], ps)
    table, a, b = s["table"], s["src"].long(), s["dst"].long()
    kv = s["kv_lens"].long()[a]
    full, part = kv // ps, kv % ps
    need = (part > 0).long()
    taken = need.cumsum(0)
    ok = (need == 0) | (taken <= freed[0])
    fresh = s["free"][(freed[0] - taken).clamp(min=0).long()]
    at = torch.arange(table.shape[1], device=DEV)[None]
    rows = table[a]
    shared = (at < full[:, None]) & ok[:, None]
    s["refs"].index_add_(0, torch.where(shared, rows, 0).view(-1), shared.int().view(-1))
    last = (at == full[:, None]) & (part > 0)[:, None]
    new = torch.where(shared, rows, torch.where(last & ok[:, None], fresh[:, None], table[b]))
    table[b] = new
    s["kv_lens"][b] = torch.where(ok, kv, s["kv_lens"][b].long()).int()
    j = torch.arange(ps, device=DEV)[None]
    has = (j < part[:, None]) & ok[:, None]
    src = torch.where(has, rows.gather(1, full[:, None].clamp(max=table.shape[1] - 1)).long() * ps + j, -1)
    dst = torch.where(has, fresh[:, None].long() * ps + j, -1)
    for C in (s["K"], s["V"]):
        _moved(C, src[has], dst[has], ps)
    used = (need * ok).sum()
    info = torch.stack([freed[0] - used, used, (~ok).sum(), shared.sum()]).int()
    return s["kv_lens"], table, s["refs"], s["free"], freed, src.int(), dst.int(), info, s["K"], s["V"]


# ---- what one pass cannot do without ----


def work(case):
    if case["kind"] == "logp":
        n = case["T"] * case["V"]
        return dict(bytes=n * (2 if case["dtype"] == "bf16" else 4) + case["T"] * (case["tokens"] * 8 + case["top"] * 8 + 8), flops=4 * n)
    Hkv, D, ps = case["Hkv"], case["D"], case["ps"]
    if case["kind"] == "fork":
        # half a page of a fork on average, read and written; lengths, table rows, the list's pages
        pages = case["kv"] / ps / 2
        tokens = case["N"] * min(ps, case["kv"]) / 2
        return dict(bytes=tokens * case["layers"] * Hkv * D * 8 + case["N"] * (pages * 20 + ps * 8 + 16) + case["B"] * 12, flops=0)
    pairs = _lengths(case)
    T = sum(n for _, n in pairs)
    if case["kind"] == "commit":
        # about two tokens of a tree have another place
        return dict(bytes=case["B"] * 2 * case["layers"] * Hkv * D * 8 + T * 24 + case["B"] * 28, flops=0)
    Hq, P = case["Hq"], case["prefix"]
    cached = P + sum(a + n for a, n in pairs)
    seen = sum(n * (P + a + 1) for a, n in pairs)
    return dict(bytes=cached * Hkv * D * 4 + T * (Hq * D * 4 + Hq * 4 + 8 + 8 * case["words"]), flops=seen * Hq * D * 4)


# ---- the definitions in 64 bits ----


def exact(case, seed):
    return {"tree": _exact_tree, "logp": _exact_logp, "commit": _exact_commit, "fork": _exact_fork}[case["kind"]](prepare(case, seed))


def _exact_tree(s):
    """request by request, a row's ancestors one after the other"""
    T, Hq, Hkv, D, P, ps, words = s["T"], s["Hq"], s["Hkv"], s["D"], s["prefix"], s["ps"], s["words"]
    out = torch.empty((T, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((T, Hq), dtype=torch.float64, device=DEV)
    parents = s["parents"].tolist()
    bits, pos = [], []

    def tokens(C, pages, n):
        rows = torch.arange(n, device=DEV)
        return C[pages[rows // ps], :, rows % ps].double()  # [n, Hkv, D]
    pk, pv = (tokens(C, s["prefix_pages"].long(), P) for C in (s["K"], s["V"]))
    for b, (n, L) in enumerate(zip(s["n_list"], s["kv_list"])):
        t = s["offs_list"][b]
        sees = torch.zeros((n, P + L), dtype=torch.bool)
        sees[:, :P + L - n] = True
        for i in range(n):
            line = []
            if n > 64 * words:
                sees[i, P + L - n:P + L - n + i + 1] = True
                pos.append(P + L - n + i)
            else:
                at = i
                while at >= 0:
                    line.append(at)
                    sees[i, P + L - n + at] = True
                    at = parents[t + at]
                pos.append(P + L - n + len(line) - 1)
            value = sum(1 << a for a in line)
            for w in range(words):
                one = value >> (64 * w) & (2 ** 64 - 1)
                bits.append(one - 2 ** 64 if one >> 63 else one)
        sees = sees.to(DEV)
        k = torch.cat([pk, tokens(s["K"], s["table"][b].long(), L)])
        v = torch.cat([pv, tokens(s["V"], s["table"][b].long(), L)])
        for h in range(Hkv):
            hs = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            q = s["Q"][t:t + n].double().view(n, Hq, D)[:, hs]
            a = (q.reshape(-1, D) @ k[:, h].t()).view(n, -1, P + L) * s["scale"]
            a.masked_fill_(~sees[:, None], -math.inf)
            z = torch.logsumexp(a, -1)
            lse[t:t + n, hs] = z
            out[t:t + n, hs] = ((a - z[..., None]).exp().view(-1, P + L) @ v[:, h]).view(n, -1, D)
    return torch.tensor(bits, device=DEV).view(T, words), _i32(pos), out.view(T, Hq * D), lse


def _exact_logp(s):
    got = [[], [], [], [], []]
    for t in range(0, s["T"], 128):
        raw = s["logits"][t:t + 128].double()
        p = torch.log_softmax(raw * s["scale"], 1)
        z = torch.logsumexp(raw * s["scale"], 1)
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :s["top"]] if s["top"] else torch.zeros((raw.shape[0], 0), dtype=torch.long, device=DEV)
        for lst, x in zip(got, (p.gather(1, s["given"][t:t + 128].long()), order.int(), p.gather(1, order), z, -(p.exp() * p).sum(1))):
            lst.append(x)
    lp, ids, best, z, h = (torch.cat(x) for x in got)
    return (lp if s["tokens"] else None), (ids if s["top"] else None), (best if s["top"] else None), z, h


def _exact_free(s, old, new, free, n_free):
    refs, ps = s["refs"].tolist(), s["ps"]
    table, dead, kept = s["table"].tolist(), set(), 0
    for b, (a, c) in enumerate(zip(old, new)):
        for j in range(-(-c // ps), -(-a // ps)):
            page = table[b][j]
            if refs[page]:
                refs[page] -= 1
                kept += 1
            else:
                dead.add(page)
    for i, page in enumerate(sorted(dead)):
        free[n_free + i] = page
    s["refs"] = _i32(refs)
    return _i32([n_free + len(dead), len(dead), kept, 0])


def _exact_moved(C, pairs, ps):
    C = C.double()
    old = C.clone()
    for a, b in pairs:
        C[:, b // ps, :, b % ps] = old[:, a // ps, :, a % ps]
    return C


def _exact_commit(s):
    parents, tokens, choices, slots = (s[k].tolist() for k in ("parents", "tokens", "choices", "slots"))
    path, src, count, following, lens, pairs = [], [], [], [], [], []
    for b, n in enumerate(s["n_list"]):
        t = s["offs_list"][b]
        line = [0]
        while True:
            nxt = [i for i in range(n) if parents[t + i] == line[-1] and tokens[t + i] == choices[t + line[-1]]]
            if not nxt:
                break
            line.append(nxt[0])
        path += line + [-1] * (n - len(line))
        src += [slots[t + i] for i in line] + [-1] * (n - len(line))
        pairs += [(slots[t + i], slots[t + k]) for k, i in enumerate(line) if i != k]
        count.append(len(line))
        following.append(choices[t + line[-1]])
        lens.append(s["kv_list"][b] - n + len(line))
    K, V = (_exact_moved(s[k], pairs, s["ps"]) for k in ("K", "V"))
    free = s["free"].tolist()
    info = _exact_free(s, s["kv_list"], lens, free, s["n_free"].item())
    return _i32(path), _i32(count), _i32(following), _i32(lens), _i32(src), K, V, s["refs"], _i32(free), info


def _exact_fork(s):
    ps, free = s["ps"], s["free"].tolist()
    kv = s["kv_lens"].tolist()
    freed = _exact_free(s, kv, s["new_lens"].tolist(), free, s["n_free"].item())
    refs, table, have = s["refs"].tolist(), s["table"].tolist(), freed[0].item()
    left, src, dst, shared = have, [], [], 0
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        full, part = divmod(kv[a], ps)
        for j in range(full):
            table[b][j] = table[a][j]
            refs[table[a][j]] += 1
            shared += 1
        kv[b] = kv[a]
        if part:
            left -= 1
            table[b][full] = free[left]
            src += [table[a][full] * ps + j for j in range(part)]
            dst += [free[left] * ps + j for j in range(part)]
        src += [-1] * (ps - part)
        dst += [-1] * (ps - part)
    pairs = [(a, b) for a, b in zip(src, dst) if a >= 0]
    K, V = (_exact_moved(s[k], pairs, ps) for k in ("K", "V"))
    return (_i32(kv), _i32(table), _i32(refs), _i32(free), freed, _i32(src).view(-1, ps), _i32(dst).view(-1, ps), _i32([left, have - left, 0, shared]), K, V)
