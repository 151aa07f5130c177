"""The operators of an attention layer that stand between the quantised projections: the pages that new
tokens get in a paged cache, the per-head norms with the position rotation and the write into that cache,
and attention over a prefix that all requests share and over every request's own tokens.

kind    one pass
slots   block table, cache slots, positions and row offsets of one step from the requests' lengths
rope    norms of query and key heads, rotation, keys and values into their pages
attn    attention of the step's rows: the shared prefix and each request's own tokens

Head layouts are those of the benchmark configurations (32 query heads on 8 or 4 key/value heads of 128
channels) and a generic one with heads of 64.
"""
import math
import random

import torch

own = False
DEV = "cuda"


def listed():
    return [
        # one decode step of a small batch whose launch is padded to 64 rows (a captured graph)
        dict(name="slots_decode_50", kind="slots", B=50, mode="decode", kv=900, T=64, ps=16, base=2048, lens=1),
        # prompts of ordinary, odd lengths
        dict(name="slots_prompts_96", kind="slots", B=96, mode="prefill", kv=300, q=420, T=0, ps=64, base=0, lens=2),
        # the largest batch: chunks of prompts beside many decoding requests, small pages
        dict(name="slots_mixed_2048", kind="slots", B=2048, mode="mixed", kv=4000, q=600, T=0, ps=16, base=777, lens=3),
        # one token of one request: latency is all there is
        dict(name="rope_decode_1", kind="rope", T=1, Hq=32, Hkv=8, D=128, rot=128, style="halves", axes=1, norm=True, ps=16, far=40000),
        # a decode batch at positions far into a long context
        dict(name="rope_decode_100", kind="rope", T=100, Hq=32, Hkv=4, D=128, rot=128, style="halves", axes=1, norm=True, ps=64, far=130000),
        # a full prefill
        dict(name="rope_prefill_8192", kind="rope", T=8192, Hq=32, Hkv=8, D=128, rot=128, style="halves", axes=1, norm=True, ps=64, far=32768),
        # image and text tokens with positions in time, height and width, neighbouring pairs, part of the head rotated
        dict(name="rope_axes_2501", kind="rope", T=2501, Hq=24, Hkv=8, D=64, rot=48, style="pairs", axes=3, norm=False, ps=32, far=5000),
        # four requests that have just left a short common prompt
        dict(name="attn_decode_4", kind="attn", B=4, mode="decode", prefix=515, kv=90, Hq=32, Hkv=8, D=128, ps=16, lens=4),
        # a decode batch behind a long system prompt
        dict(name="attn_decode_64", kind="attn", B=64, mode="decode", prefix=8192, kv=700, Hq=32, Hkv=8, D=128, ps=64, lens=5),
        # the largest decode batch, long own contexts
        dict(name="attn_decode_256", kind="attn", B=256, mode="decode", prefix=32700, kv=2000, Hq=32, Hkv=4, D=128, ps=64, lens=6),
        # chunks of prompts in the same step as decoding requests
        dict(name="attn_mixed_40", kind="attn", B=40, mode="mixed", prefix=4096, kv=1500, q=1100, Hq=32, Hkv=8, D=128, ps=32, lens=7),
        # no common prefix, small heads, a few requests with long contexts
        dict(name="attn_decode_12_long", kind="attn", B=12, mode="decode", prefix=0, kv=30000, Hq=24, Hkv=8, D=64, ps=128, lens=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["slots", "rope", "rope", "attn", "attn", "attn"])
    ps = rng.choice([16, 32, 64, 128])
    lens = rng.randrange(100, 10 ** 6)
    if kind == "slots":
        mode = rng.choice(["decode", "prefill", "mixed"])
        B = _log_int(rng, 1, 2000)
        q = min(_log_int(rng, 2, 4000), 200000 // B)
        T = B + rng.randrange(0, 64) if mode == "decode" else 0
        return dict(kind=kind, B=B, mode=mode, kv=_log_int(rng, 1, 4000), q=max(q, 2), T=T, ps=ps, base=rng.choice([0, 0, _log_int(rng, 1, 30000)]),
                    lens=lens)
    Hq, Hkv, D = rng.choice([(32, 8, 128), (32, 4, 128), (24, 8, 64), (12, 12, 64), (8, 1, 128), (40, 8, 128), (28, 4, 128)])
    if kind == "rope":
        rot = rng.choice([D, D, D, D // 2, 3 * D // 4])
        T = _log_int(rng, 1, 8192 * 40 // (Hq + Hkv) if D * (Hq + Hkv) > 5120 else 8192)
        return dict(kind=kind, T=T, Hq=Hq, Hkv=Hkv, D=D, rot=rot, style=rng.choice(["halves", "halves", "pairs"]), axes=rng.choice([1, 1, 2, 3]),
                    norm=rng.random() < 0.7, ps=ps, far=_log_int(rng, 100, 130000))
    mode = rng.choice(["decode", "decode", "mixed", "prefill"])
    prefix = rng.choice([0, _log_int(rng, 16, 32000), _log_int(rng, 16, 32000)])
    if mode == "decode":
        B = _log_int(rng, 1, 256)
        kv = min(_log_int(rng, 4, 30000), 500000 // B)
        return dict(kind=kind, B=B, mode=mode, prefix=prefix, kv=kv, Hq=Hq, Hkv=Hkv, D=D, ps=ps, lens=lens)
    B = _log_int(rng, 1, 40)
    q = min(_log_int(rng, 8, 1100), (2000 if mode == "prefill" else 4000) // B + 2)
    return dict(kind=kind, B=B, mode=mode, prefix=min(prefix, 4096), kv=_log_int(rng, 4, 1500), q=q, Hq=Hq, Hkv=Hkv, D=D, ps=ps, lens=lens)


# ---- lengths: the case's own, so that every seed has the same work; a seed deals them to the requests ----


def _lengths(case):
    """(tokens a request has cached before the step, tokens of the step), one pair a request"""
    rng = random.Random(case["lens"])
    out = []
    for b in range(case["B"]):
        kv = rng.randint(0, case["kv"]) if b % 8 else case["kv"]
        if case["mode"] == "decode":
            q = 1
        elif case["mode"] == "prefill":
            q = rng.randint(1, case["q"])
            kv = kv if rng.random() < 0.5 else 0
        else:
            q = rng.randint(case["q"] // 4 + 1, case["q"]) if b % 10 == 3 or b == 0 else 1
        out.append((kv, q))
    return out


def _deal(case, seed):
    pairs = _lengths(case)
    random.Random(seed * 7919 + 1).shuffle(pairs)
    return [a for a, _ in pairs], [b for _, b in pairs]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *size, std=1.0):
    """bf16 values, made in pieces: a long cache is large"""
    out = torch.empty(size, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    step = 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device=DEV) * std
    return out


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _sections(case):
    """how many of the rotated pairs belong to each axis"""
    half, n = case["rot"] // 2, case["axes"]
    if n == 1:
        return [half]
    first = half // 4 if n == 3 else half // 3
    rest = half - first
    return [first, rest] if n == 2 else [first, rest // 2, rest - rest // 2]


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    ps = case["ps"]
    if case["kind"] == "slots":
        kv, q = _deal(case, seed)
        B = case["B"]
        T = case["T"] or sum(q)
        old = [-(-a // ps) for a in kv]
        new = [-(-(a + b) // ps) for a, b in zip(kv, q)]
        total = sum(new) + 37
        perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        table = torch.full((B, max(new) + 3), -1, dtype=torch.int32, device=DEV)
        have = _i32(old)[:, None] > torch.arange(table.shape[1], device=DEV)[None]
        table[have] = perm[:sum(old)]
        s.update(T=T, kv_lens=_i32(kv), q_lens=_i32(q), table=table, free=perm[sum(old):].contiguous(), n_free=_i32([total - sum(old)]))
        return s
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["kind"] == "rope":
        T, rot, far = case["T"], case["rot"], case["far"]
        n_pos = far + 1
        inv = 1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
        ang = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * inv
        n_pages = -(-T // ps) + 5
        slots = (torch.randperm(n_pages, generator=g, device=DEV)[:, None] * ps + torch.arange(ps, device=DEV)).view(-1)[3:3 + T]
        pos = torch.randint(0, n_pos, (case["axes"], T), generator=g, device=DEV, dtype=torch.int32)
        s.update(x=_randn(g, T, (Hq + 2 * Hkv) * D), table=torch.cat([ang.cos(), ang.sin()], 1).float(), pos=pos, slots=slots.to(torch.int32),
                 gq=(1 + 0.3 * torch.randn(D, generator=g, device=DEV)).bfloat16() if case["norm"] else None,
                 gk=(1 + 0.3 * torch.randn(D, generator=g, device=DEV)).bfloat16() if case["norm"] else None,
                 K=_randn(g, n_pages, Hkv, ps, D), V=_randn(g, n_pages, Hkv, ps, D), sections=_sections(case))
        return s
    kv0, q = _deal(case, seed)
    kv = [a + b for a, b in zip(kv0, q)]  # the step's tokens are in the cache by now
    B, T, P = case["B"], sum(q), case["prefix"]
    pages = [-(-a // ps) for a in kv]
    n_prefix = -(-P // ps)
    n_pages = sum(pages) + n_prefix + 2
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, max(pages)), -1, dtype=torch.int32, device=DEV)
    table[_i32(pages)[:, None] > torch.arange(table.shape[1], device=DEV)[None]] = perm[n_prefix:n_prefix + sum(pages)]
    offs = [0]
    for n in q:
        offs.append(offs[-1] + n)
    s.update(T=T, q_list=q, kv_list=kv, Q=_randn(g, T, Hq * D, std=1.5), K=_randn(g, n_pages, Hkv, ps, D), V=_randn(g, n_pages, Hkv, ps, D),
             prefix_pages=perm[:n_prefix].contiguous(), table=table, kv_lens=_i32(kv), q_offsets=_i32(offs), scale=D ** -0.5)
    if own:
        import paper_2604_12782_amd as osc
        n = osc.osc_prefix_attention_workspace_bytes(T, B, Hq, Hkv, D, P)
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----


def run(s):
    return {"slots": _slots, "rope": _rope, "attn": _attn}[s["kind"]](s)


def _slots(s):
    if own:
        import paper_2604_12782_amd as osc
        lens, offs, pos, slots, info = osc.osc_page_slots(s["kv_lens"], s["q_lens"], s["free"], s["n_free"], s["table"], s["ps"], s["T"], s["base"])
        return s["table"], lens, offs, pos, slots, info
    ps, table, free = s["ps"], s["table"], s["free"]
    kv, q = s["kv_lens"].long(), s["q_lens"].long()
    old = (kv + ps - 1) // ps
    new = (kv + q + ps - 1) // ps
    fits = new <= table.shape[1]
    need = torch.where(fits, new - old, 0)
    incl = need.cumsum(0)
    ok = fits & ((need == 0) | (incl <= s["n_free"]))
    offs = torch.cat([q.new_zeros(1), q.cumsum(0)])
    t = torch.arange(s["T"], device=DEV)
    real = t < offs[-1]
    req = (torch.searchsorted(offs, t, right=True) - 1).clamp(max=kv.numel() - 1)
    p = kv[req] + t - offs[req]
    page_i = (p // ps).clamp(max=table.shape[1] - 1)
    there = table[req, page_i].long()
    taken = (incl - need)[req] + page_i - old[req]
    fresh = free[(s["n_free"] - 1 - taken).clamp(0, free.numel() - 1)].long()
    good = real & ok[req]
    page = torch.where(good & (page_i >= old[req]), fresh, there)
    req_w = torch.where(real, req, kv.numel() - 1)
    last = table.shape[1] - 1
    table[req_w, torch.where(real, page_i, last)] = torch.where(real, page, table[-1, last].long()).int()
    slots = torch.where(good, page * ps + p % ps, -1)
    pos = torch.where(real, s["base"] + p, -1)
    used = torch.where(ok, need, 0).sum()
    info = torch.stack([s["n_free"][0] - used, used, (~ok).sum(), offs[-1]])
    return table, torch.where(ok, kv + q, kv).int(), offs.int(), pos.int(), slots.int(), info.int()


def _rotate(x, cos, sin, rot, style):
    """x [T, H, D] in 32 bits; cos, sin [T, 1, rot/2]"""
    if style == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., rot:]], -1)


def _rope(s):
    Hq, Hkv, D, rot, ps = s["Hq"], s["Hkv"], s["D"], s["rot"], s["ps"]
    if own:
        import paper_2604_12782_amd as osc
        style = osc.OSC_ROPE_HALVES if s["style"] == "halves" else osc.OSC_ROPE_PAIRS
        y = osc.osc_qk_norm_rope(s["x"], Hq, Hkv, D, s["table"], s["pos"], s["slots"], s["K"], s["V"], s["gq"], s["gk"], 1e-6, rot, style, s["sections"])
        return y, s["K"], s["V"]
    T = s["T"]
    x = s["x"].view(T, Hq + 2 * Hkv, D)
    axis = torch.cat([torch.full((n,), a, device=DEV) for a, n in enumerate(s["sections"])])
    pair = torch.arange(rot // 2, device=DEV)
    at = s["pos"].long()[axis].t()  # [T, rot/2]
    cos = s["table"][at, pair][:, None]
    sin = s["table"][at, pair + rot // 2][:, None]

    def head(h, gamma):
        h = h.float()
        if gamma is not None:
            h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * gamma.float()
        return _rotate(h, cos, sin, rot, s["style"]).bfloat16()
    y = head(x[:, :Hq], s["gq"]).reshape(T, Hq * D)
    page, off = s["slots"].long() // ps, s["slots"].long() % ps
    s["K"][page, :, off] = head(x[:, Hq:Hq + Hkv], s["gk"])
    s["V"][page, :, off] = x[:, Hq + Hkv:]
    return y, s["K"], s["V"]


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
    """rows 0..n-1 of a request (or of the prefix) from its pages: [..., Hkv, n, D] in 32 bits"""
    x = C[pages].float()  # [..., pages, Hkv, ps, D]
    x = x.transpose(-4, -3).flatten(-3, -2)
    return x[..., :n, :]


def _attn(s):
    T, Hq, Hkv, D, P = s["T"], s["Hq"], s["Hkv"], s["D"], s["prefix"]
    if own:
        import paper_2604_12782_amd as osc
        return osc.osc_prefix_attention(s["Q"], Hq, Hkv, D, s["K"], s["V"], s["prefix_pages"], P, s["table"], s["kv_lens"], s["q_offsets"], s["scale"],
                                        want_lse=True, workspace=s["workspace"])
    G, B, scale = Hq // Hkv, s["B"], s["scale"]
    q = s["Q"].float().view(T, Hkv, G, D).transpose(0, 1)  # [Hkv, T, G, D]
    if max(s["q_list"]) == 1:
        n = max(s["kv_list"])
        pages = s["table"].long().clamp(min=0)
        k, v = _cached(s["K"], pages, n), _cached(s["V"], pages, n)
        mask = torch.arange(n, device=DEV) < s["kv_lens"][:, None]
        num, den, top = _part(q.transpose(0, 1), k, v, scale, mask[:, None, None])
        acc = [x.transpose(0, 1) for x in (num, den, top)]  # [Hkv, T, G, .]
    else:
        parts, t = [], 0
        for b in range(B):
            n, L = s["q_list"][b], s["kv_list"][b]
            pages = s["table"][b, :-(-L // s["ps"])].long()
            k, v = _cached(s["K"], pages, L), _cached(s["V"], pages, L)
            mask = torch.arange(L, device=DEV) <= (L - n + torch.arange(n, device=DEV))[:, None]
            x = _part(q[:, t:t + n].reshape(Hkv, n * G, D), k, v, scale, mask.repeat_interleave(G, 0))
            parts.append([y.view(Hkv, n, G, -1) for y in x])
            t += n
        acc = [torch.cat([p[i] for p in parts], 1) for i in range(3)]
    if P:
        pages = s["prefix_pages"].long()
        k, v = _cached(s["K"], pages, P), _cached(s["V"], pages, P)
        heads = [_part(q[h].reshape(T * G, D), k[h], v[h], scale) for h in range(Hkv)]
        pre = [torch.stack([p[i] for p in heads]).view(Hkv, T, G, -1) for i in range(3)]
        acc = _join(acc, pre)
    num, den, top = acc
    out = (num / den).transpose(0, 1).reshape(T, Hq * D).bfloat16()
    lse = (top + torch.log(den)).transpose(0, 1).reshape(T, Hq)
    return out, lse


# ---- what one pass cannot do without ----


def work(case):
    if case["kind"] == "slots":
        pairs = _lengths(case)
        ps = case["ps"]
        T = case["T"] or sum(q for _, q in pairs)
        new = sum(-(-(a + b) // ps) - -(-a // ps) for a, b in pairs)
        # lengths in and out, offsets; a free page read and its entry written; the page of a partly filled last one; slot and position a row
        return dict(bytes=case["B"] * 16 + new * 8 + case["B"] * 4 + T * 8, flops=0)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["kind"] == "rope":
        T, rot = case["T"], case["rot"]
        rows = min(T * case["axes"], case["far"] + 1)
        heads = Hq + 2 * Hkv
        return dict(bytes=T * heads * D * 4 + rows * rot * 4 + T * (case["axes"] + 1) * 4, flops=T * (Hq + Hkv) * (D * (4 if case["norm"] else 0) + rot * 3))
    pairs = _lengths(case)
    T = sum(q for _, q in pairs)
    cached = case["prefix"] + sum(a + b for a, b in pairs)
    seen = T * case["prefix"] + sum(q * a + q * (q + 1) // 2 for a, q in pairs)
    return dict(bytes=cached * Hkv * D * 4 + T * Hq * D * 4 + T * Hq * 4, flops=seen * Hq * D * 4)


# ---- the definitions in 64 bits ----


def exact(case, seed):
    return {"slots": _exact_slots, "rope": _exact_rope, "attn": _exact_attn}[case["kind"]](prepare(case, seed))


def _exact_slots(s):
    """request by request, page by page"""
    ps, T = s["ps"], s["T"]
    table = s["table"].tolist()
    free = s["free"].tolist()[:s["n_free"].item()]
    lens, offs, pos, slots, refused, top = [], [0], [], [], 0, len(free)
    asked = 0
    for b, (kv, q) in enumerate(zip(s["kv_lens"].tolist(), s["q_lens"].tolist())):
        have, want = math.ceil(kv / ps), math.ceil((kv + q) / ps)
        served = want <= len(table[b])
        if served:
            first = asked
            asked += want - have
            served = want == have or asked <= len(free)
        if served:
            for j in range(have, want):
                table[b][j] = free[len(free) - 1 - first - (j - have)]
            top -= want - have
        for p in range(kv, kv + q):
            pos.append(s["base"] + p)
            slots.append(table[b][p // ps] * ps + p % ps if served else -1)
        lens.append(kv + q if served else kv)
        refused += not served
        offs.append(offs[-1] + q)
    pad = T - len(pos)
    return (_i32(table), _i32(lens), _i32(offs), _i32((pos + [-1] * pad)[:T]), _i32((slots + [-1] * pad)[:T]),
            _i32([top, len(free) - top, refused, offs[-1]]))


def _exact_rope(s):
    Hq, Hkv, D, rot, ps, T = s["Hq"], s["Hkv"], s["D"], s["rot"], s["ps"], s["T"]
    x = s["x"].double().view(T, Hq + 2 * Hkv, D)
    z = x.clone()
    for lo, hi, gamma in ((0, Hq, s["gq"]), (Hq, Hq + Hkv, s["gk"])):
        if gamma is not None:
            z[:, lo:hi] = x[:, lo:hi] / (x[:, lo:hi].pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * gamma.double()
    y = z.clone()
    i = 0
    for a, n in enumerate(s["sections"]):
        for i in range(i, i + n):
            c = s["table"][s["pos"][a].long(), i].double()[:, None]
            d = s["table"][s["pos"][a].long(), rot // 2 + i].double()[:, None]
            u, w = (i, i + rot // 2) if s["style"] == "halves" else (2 * i, 2 * i + 1)
            heads = slice(0, Hq + Hkv)
            y[:, heads, u] = z[:, heads, u] * c - z[:, heads, w] * d
            y[:, heads, w] = z[:, heads, u] * d + z[:, heads, w] * c
        i += 1
    K, V = s["K"].double(), s["V"].double()
    for C, lo in ((K, Hq), (V, Hq + Hkv)):
        rows = C.transpose(1, 2).reshape(-1, Hkv, D)
        rows[s["slots"].long()] = y[:, lo:lo + Hkv]
        C.copy_(rows.view(C.shape[0], ps, Hkv, D).transpose(1, 2))
    return y[:, :Hq].reshape(T, Hq * D), K, V


def _exact_attn(s):
    Hq, Hkv, D, P, ps = s["Hq"], s["Hkv"], s["D"], s["prefix"], s["ps"]
    out = torch.empty((s["T"], Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((s["T"], Hq), dtype=torch.float64, device=DEV)

    def tokens(C, pages, n):
        rows = torch.arange(n, device=DEV)
        return C[pages[rows // ps], :, rows % ps].double()  # [n, Hkv, D]
    pk, pv = (tokens(C, s["prefix_pages"].long(), P) for C in (s["K"], s["V"]))
    t = 0
    for b, (n, L) in enumerate(zip(s["q_list"], s["kv_list"])):
        k = torch.cat([pk, tokens(s["K"], s["table"][b].long(), L)])
        v = torch.cat([pv, tokens(s["V"], s["table"][b].long(), L)])
        for i in range(0, n, 256):
            rows = range(t + i, t + min(i + 256, n))
            last = P + L - n + torch.arange(i, min(i + 256, n), device=DEV)
            sees = torch.arange(P + L, device=DEV)[None] <= last[:, None]
            for h in range(Hkv):
                hs = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
                q = s["Q"][rows.start:rows.stop].double().view(len(rows), Hq, D)[:, hs]
                a = (q.reshape(-1, D) @ k[:, h].t()).view(len(rows), -1, P + L) * s["scale"]
                a.masked_fill_(~sees[:, None], -math.inf)
                z = torch.logsumexp(a, -1)
                lse[rows.start:rows.stop, hs] = z
                out[rows.start:rows.stop, hs] = ((a - z[..., None]).exp().view(-1, P + L) @ v[:, h]).view(len(rows), -1, D)
        t += n
    return out.view(s["T"], Hq * D), lse
