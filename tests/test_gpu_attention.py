"""Cache pages, per-head norms with rotation, and attention behind a shared prefix, on the GPU against their plain
forms in 64 bits (oracle/attention.py).

Tolerances.  bf16 results are rounded once: 2^-8 of the value.  Norm and rotation are about 30 single-precision
operations on terms no larger than the pair's length: 2^-19 of it.  Attention weights are rounded to bf16 before
the second product: 2^-8 of the weighted average of |v|; scores are sums of D products (D 2^-24 of the sum of their
magnitudes, times the scale), and an error of a score is a relative error of its weight."""
import numpy as np
import pytest
import torch

from oracle import attention as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def osc():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_12782_amd as m
    m.lib()
    return m


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


# ---- pages and slots ----------------------------------------------------------------------------------------------


def check_slots(osc, kv, q, ps, n_pool, n_free, width, T, base=0, seed=0):
    gen = np.random.default_rng(seed)
    B = len(kv)
    pages = gen.permutation(n_pool + B * width)
    free, table = pages[:n_pool], pages[n_pool:].reshape(B, width)
    want = ref.page_slots(kv, q, ps, free, n_free, table, T, base)
    d_table = i32(table)
    got = osc.osc_page_slots(i32(kv), i32(q), i32(free), i32([n_free]), d_table, ps, T, base)
    for name, g, w in zip(("lengths", "offsets", "positions", "slots", "info", "table"), (*got, d_table), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    return got


@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 255, 256, 257, 1025])
def test_slots(osc, B, ps):
    gen = np.random.default_rng(B * 7 + ps)
    kv, q = gen.integers(0, 3 * ps, B), gen.integers(0, 2 * ps, B)
    kv[gen.random(B) < 0.3] = ps  # full pages
    q[gen.random(B) < 0.3] = 1
    q[gen.random(B) < 0.2] = 0
    check_slots(osc, kv, q, ps, 3 * B + 5, 3 * B + 5, 6, int(q.sum()), 11)
    check_slots(osc, kv, q, ps, 3 * B + 5, 3 * B + 2, 6, int(q.sum()) + 77, 0)  # padded rows; not the whole list is free


def test_slots_refused(osc):
    kv, q = [0, 15, 16, 40, 5, 0, 3], [33, 1, 1, 200, 11, 0, 30]
    for n_free in range(0, 9):  # the fourth asks for more than its row of the table; others run out of pages
        got = check_slots(osc, kv, q, 16, 9, n_free, 5, sum(q), 3, seed=n_free)
        assert got[4][2].item() >= 1
    check_slots(osc, kv, q, 16, 9, 10 ** 6, 5, sum(q))  # more free than the list holds
    check_slots(osc, kv, q, 16, 9, -4, 5, sum(q))
    check_slots(osc, [-5, 7], [3, -2], 16, 4, 4, 2, 3)  # negative lengths count as none
    # sums past 32 bits: that request is refused, and the row offsets stop at the largest number
    lens, offs, pos, slots, info = osc.osc_page_slots(i32([2 ** 31 - 1, 5]), i32([2 ** 31 - 1, 9]), i32([3, 2]), i32([2]), i32([[0, 0], [1, 0]]), 16, 50)
    assert lens.tolist() == [2 ** 31 - 1, 14] and offs.tolist() == [0, 2 ** 31 - 1, 2 ** 31 - 1] and info.tolist() == [2, 0, 1, 2 ** 31 - 1]
    assert (slots == -1).all()


def test_slots_most_requests(osc):
    gen = np.random.default_rng(5)
    kv, q = gen.integers(0, 40, 8192), gen.integers(0, 9, 8192)
    check_slots(osc, kv, q, 16, 8192, 8192, 4, int(q.sum()))


def test_slots_step_by_step(osc):
    """a serving loop: lengths, free count and table go from step to step on the device"""
    B, ps, width, n_pool = 5, 16, 8, 30
    lens = [i32([0, 3, 16, 0, 31]), torch.empty(B, dtype=torch.int32, device=DEV)]
    table = i32(100 + np.arange(B * width).reshape(B, width))
    free, n_free = i32(np.arange(n_pool)[::-1].copy()), i32([n_pool])
    w_lens, w_table, w_free = lens[0].cpu().numpy(), table.cpu().numpy(), n_pool
    gen = np.random.default_rng(3)
    for step in range(12):
        q = gen.integers(0, 14, B)
        T = int(q.sum())
        want = ref.page_slots(w_lens, q, ps, free.cpu().numpy(), w_free, w_table, T, 100)
        kv, offs, pos, slots, info = osc.osc_page_slots(lens[step % 2], i32(q), free, n_free, table, ps, T, 100)
        for g, w in zip((kv, offs, pos, slots, info, table), want):
            assert np.array_equal(g.cpu().numpy(), w), step
        lens[1 - step % 2], n_free = kv, info[:1].clone()
        w_lens, w_table, w_free = want[0], want[5], want[4][0]


@pytest.mark.parametrize("T", [0, 1, 300])
def test_slots_no_requests(osc, T):
    """an idle step of a launch padded to T rows: every row is padding, nothing is taken"""
    none, table = i32([]), torch.empty((0, 4), dtype=torch.int32, device=DEV)
    for n_pool, n_free, left in ((9, 7, 7), (9, 12, 9), (9, -3, 0), (0, 5, 0)):
        outs = [torch.full((n,), 77, dtype=torch.int32, device=DEV) for n in (0, 1, T, T, 4)]
        for out in (tuple(outs), None):
            lens, offs, pos, slots, info = osc.osc_page_slots(none, none, i32(np.arange(n_pool)), i32([n_free]), table, 16, T, 5, out=out)
            assert lens.numel() == 0 and offs.tolist() == [0] and info.tolist() == [left, 0, 0, 0]
            assert pos.tolist() == slots.tolist() == [-1] * T


@pytest.mark.parametrize("B", [1, 5, 300, 1500, 2500])
def test_slots_fewer_rows_than_tokens(osc, B):
    """tokens past T have no row; their requests' pages are dealt and entered all the same, so the next step finds them"""
    gen = np.random.default_rng(B)
    kv, q = gen.integers(0, 70, B), gen.integers(0, 60, B)
    kv[gen.random(B) < 0.3] = 32
    q[0] = 45  # three pages in one request
    pages = sum(-(-(a + b) // 16) - -(-a // 16) for a, b in zip(kv.tolist(), q.tolist()))
    for T in (0, 1, 16, int(q.sum()) // 2, int(q.sum()) - 1):
        check_slots(osc, kv, q, 16, pages + 3, pages + 3, 9, T, 7, seed=T)
        check_slots(osc, kv, q, 16, pages + 3, pages // 2, 6, T, 7, seed=T)  # some are refused, for want of pages or of room in the table


def test_slots_of_pages_that_no_cache_has(osc):
    """a page number that is negative, or whose slots 31 bits cannot hold, gives slot -1, not another page's slot"""
    for ps in (16, 256):
        lim = 2 ** 31 // ps
        bad = [lim, -lim, -1, 2 ** 31 - 1, -2 ** 31, lim + 1, 2 * lim % 2 ** 31]
        kv, q = [3] * len(bad), [2] * len(bad)
        _, _, pos, slots, _ = osc.osc_page_slots(i32(kv), i32(q), i32([]), i32([0]), i32([[b] for b in bad]), ps, 2 * len(bad))
        assert pos.tolist() == [3, 4] * len(bad)
        want = [b * ps + r if 0 <= b < lim else -1 for b in bad for r in (3, 4)]
        assert slots.tolist() == want
        fresh = osc.osc_page_slots(i32([0] * len(bad)), i32(q), i32(bad[::-1]), i32([len(bad)]), i32([[5]] * len(bad)), ps, 2 * len(bad))
        assert fresh[3].tolist() == [b * ps + r if 0 <= b < lim else -1 for b in bad for r in (0, 1)]
        assert osc.osc_page_slots(i32([3]), i32([1]), i32([]), i32([0]), i32([[lim - 1]]), ps, 1)[3].tolist() == [(lim - 1) * ps + 3]
    gen = np.random.default_rng(9)
    table = gen.integers(-2 ** 31, 2 ** 31, (40, 3))
    kv, q = gen.integers(1, 17, 40), gen.integers(0, 15, 40)
    want = ref.page_slots(kv, q, 16, np.arange(40), 40, table, int(q.sum()))
    assert np.array_equal(osc.osc_page_slots(i32(kv), i32(q), i32(np.arange(40)), i32([40]), i32(table), 16, int(q.sum()))[3].cpu().numpy(), want[3])


# ---- norms, rotation, cache ------------------------------------------------------------------------------------------


def test_rope_table(osc):
    for base, rot, n in ((10000.0, 128, 300), (1e6, 64, 77), (5e5, 8, 70000)):
        got, want = f64(osc.osc_rope_table(base, rot, n)), ref.rope_angles(base, rot, n)
        assert np.abs(got - want).max() <= 2.0 ** -24 + n * 2.0 ** -50  # one rounding, and the angle's own in double


def check_rope(osc, T, Hq, Hkv, D, rot, style, axes, norm, ps=16, pad=0, seed=0, cache=True, inplace=False, sections=None, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    width = (Hq + 2 * Hkv) * D
    x = (torch.randn(T, width + pad, generator=g) * scale).bfloat16().to(DEV)[:, :width]
    gq, gk = ((1 + 0.3 * torch.randn(D, generator=g)).bfloat16().to(DEV) for _ in range(2)) if norm else (None, None)
    n_pos = 501
    cs = osc.osc_rope_table(10000.0, rot, n_pos) if rot else torch.zeros((n_pos, 0), device=DEV)
    pos = torch.randint(0, n_pos, (axes, T), generator=g, dtype=torch.int32)
    half = rot // 2
    if sections is None:
        sections = [half] if axes == 1 else [half // 3, half - half // 3] if axes == 2 else [half // 4, half // 3, half - half // 4 - half // 3]
    n_pages = T // ps + 3
    slots = torch.randperm(n_pages * ps, generator=g)[:T].int()
    out_of_range = torch.zeros(T, dtype=torch.bool)
    skip = torch.zeros(T, dtype=torch.bool)
    if T > 4:
        pos[axes - 1, 1], pos[0, 3] = n_pos, -1
        out_of_range[1] = out_of_range[3] = True
        slots[2], slots[4] = -1, n_pages * ps
        skip[2] = skip[4] = True
    K, V = (torch.randn(n_pages, Hkv, ps, D, generator=g).bfloat16().to(DEV) for _ in range(2))
    want_K, want_V = f64(K), f64(V)
    x64, pos_n = f64(x).reshape(T, Hq + 2 * Hkv, D), pos.clamp(0, n_pos - 1).numpy()
    cs64 = f64(cs)
    args = (1e-6, cs64, pos_n, sections, rot, style == osc.OSC_ROPE_PAIRS)
    wq, sq = ref.head_rope(x64[:, :Hq], None if gq is None else f64(gq), *args)
    wk, sk = ref.head_rope(x64[:, Hq:Hq + Hkv], None if gk is None else f64(gk), *args)
    wq[out_of_range.numpy()] = 0
    size_K = np.zeros_like(want_K)
    for t in range(T):
        if not (out_of_range[t] or skip[t]):
            s = int(slots[t])
            want_K[s // ps, :, s % ps], want_V[s // ps, :, s % ps], size_K[s // ps, :, s % ps] = wk[t], x64[t, Hq + Hkv:], sk[t]
    out = x[:, :Hq * D] if inplace else None
    y = osc.osc_qk_norm_rope(x, Hq, Hkv, D, cs, pos.to(DEV) if axes > 1 else pos[0].to(DEV), slots.to(DEV) if cache else None, K if cache else None,
                             V if cache else None, gq, gk, 1e-6, rot, style, sections, out)
    err = np.abs(f64(y).reshape(T, Hq, D) - wq)
    assert (err <= 2.0 ** -8 * np.abs(wq) + 2.0 ** -19 * sq).all()
    if cache:
        assert (np.abs(f64(K) - want_K) <= (size_K > 0) * 2.0 ** -8 * np.abs(want_K) + 2.0 ** -19 * size_K).all()
        assert np.array_equal(f64(V), want_V)
    return y


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 32, 8, 128), (7, 5, 5, 64), (65, 4, 1, 128), (33, 8, 2, 64), (130, 3, 1, 64), (300, 32, 4, 128)])
@pytest.mark.parametrize("style", [0, 1])
def test_rope(osc, T, Hq, Hkv, D, style):
    for axes, norm in ((1, True), (1, False), (3, True), (2, False)):
        for rot in (D, D // 2, 24):
            check_rope(osc, T, Hq, Hkv, D, rot, style, axes, norm, ps=16 << (T % 5), seed=T + axes + rot)


def test_rope_forms(osc):
    check_rope(osc, 9, 4, 2, 128, 128, 0, 1, True, pad=24)             # strided rows
    check_rope(osc, 9, 4, 2, 128, 128, 0, 1, True, cache=False)        # queries alone
    check_rope(osc, 9, 4, 2, 128, 128, 0, 1, True, inplace=True)       # over the projection's own queries
    check_rope(osc, 9, 4, 2, 64, 0, 0, 1, True)                        # nothing turned
    check_rope(osc, 9, 4, 2, 64, 64, 1, 3, True, sections=[0, 32, 0])  # empty axes
    check_rope(osc, 9, 4, 2, 64, 64, 0, 2, True, sections=[5, 27])
    check_rope(osc, 9, 4, 2, 128, 64, 0, 1, True, scale=2.0 ** 40)     # squares far above, and below, what 16 bits hold
    check_rope(osc, 9, 4, 2, 128, 64, 1, 1, True, scale=2.0 ** -7)
    check_rope(osc, 2000, 6, 2, 128, 128, 0, 1, True, ps=64)
    check_rope(osc, 9, 4, 2, 128, 128, 0, 3, True, sections=[16, 24, 24])  # whole groups of four pairs an axis
    for style in (0, 1):  # several groups of heads a wavefront, the last one not full
        check_rope(osc, 2300, 25, 5, 128, 128, style, 1, True, ps=64)
        check_rope(osc, 4200, 25, 5, 64, 48, style, 3, True, ps=32)
        check_rope(osc, 4200, 25, 5, 64, 64, style, 3, False, ps=32, sections=[8, 12, 12])


# ---- attention ---------------------------------------------------------------------------------------------------------


def make(seed, B, P, kv, n, Hq, Hkv, D, ps, std=1.5, extra_cols=0):
    """a cache that holds NaN wherever no token is"""
    g = torch.Generator().manual_seed(seed)
    pages = [-(-a // ps) for a in kv]
    n_prefix = -(-P // ps)
    n_pages = n_prefix + sum(pages) + 2
    perm = torch.randperm(n_pages, generator=g)
    K, V = (torch.full((n_pages, Hkv, ps, D), float("nan")) for _ in range(2))
    table = torch.full((B, max(pages + [1]) + 1), 10 ** 9, dtype=torch.int32)
    at = n_prefix

    def fill(pg, L):
        for j in range(L):
            K[pg[j // ps], :, j % ps] = torch.randn(Hkv, D, generator=g)
            V[pg[j // ps], :, j % ps] = torch.randn(Hkv, D, generator=g) + 0.3
    fill(perm, P)
    for b in range(B):
        pg = perm[at:at + pages[b]]
        at += pages[b]
        table[b, :pages[b]] = pg.int()
        fill(pg, kv[b])
    T = sum(n)
    Q = (torch.randn(T, Hq * D + extra_cols, generator=g) * std).bfloat16()
    offs = np.concatenate([[0], np.cumsum(n)])
    return dict(Q=Q.to(DEV)[:, :Hq * D], K=K.bfloat16().to(DEV), V=V.bfloat16().to(DEV), prefix=perm[:n_prefix].int().to(DEV), P=P, table=table.to(DEV),
                kv=i32(kv), offs=i32(offs), Hq=Hq, Hkv=Hkv, D=D, scale=D ** -0.5)


def call(osc, s, **kw):
    return osc.osc_prefix_attention(s["Q"], s["Hq"], s["Hkv"], s["D"], s["K"], s["V"], s["prefix"], s["P"], s["table"], s["kv"], s["offs"], s["scale"],
                                    want_lse=True, **kw)


def check_attention(osc, s, got=None):
    o, lse = call(osc, s) if got is None else got
    T, D, scale = s["Q"].shape[0], s["D"], s["scale"]
    wo, wl, av, big = ref.prefix_attention(f64(s["Q"]).reshape(T, s["Hq"], D), f64(s["K"]), f64(s["V"]), s["prefix"].cpu().numpy(), s["P"],
                                           s["table"].cpu().numpy(), s["kv"].cpu().numpy(), s["offs"].cpu().numpy(), scale)
    n = s["P"] + int(s["kv"].max())
    score = scale * (D + 4) * 2.0 ** -24 * big  # of a score
    err = np.abs(f64(o).reshape(T, s["Hq"], D) - wo)
    assert (err <= 2.0 ** -8 * np.abs(wo) + (2.0 ** -8 + 2 * score[..., None] + 2.0 ** -18) * av).all(), (err / (av + 1e-30)).max()
    empty = np.isinf(wl)
    assert np.array_equal(np.isinf(f64(lse)), empty)
    tol = score + 2.0 ** -21 * (np.abs(np.where(empty, 0, wl)) + scale * big) + (n + 8) * 2.0 ** -24
    assert (np.abs(np.where(empty, 0, f64(lse)) - np.where(empty, 0, wl)) <= tol).all()
    return o, lse


HEADS = [(4, 1, 128), (32, 8, 128), (6, 2, 64), (3, 3, 64), (12, 1, 128), (40, 8, 64), (48, 1, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [0, 1, 16, 31, 33, 250])
def test_attention_decode(osc, Hq, Hkv, D, P):
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 130]
    ps = 16 << ((Hq + P) % 5)
    check_attention(osc, make(P + Hq, len(kv), P, kv, [1] * len(kv), Hq, Hkv, D, ps))


@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("P", [0, 40, 129])
def test_attention_ragged(osc, ps, P):
    """prompts, chunks of prompts, single tokens and idle requests in one step"""
    n = [5, 1, 0, 33, 1, 70, 8, 0, 17, 130]
    kv = [5, 90, 12, 40, 1, 170, 8, 0, 300, 133]
    check_attention(osc, make(ps + P, len(n), P, kv, n, 8, 2, 128, ps))
    check_attention(osc, make(ps + P + 1, len(n), P, kv, n, 3, 1, 64, ps, extra_cols=40))


@pytest.mark.parametrize("D", [64, 128])
def test_attention_rows_that_see_nothing(osc, D):
    s = make(1, 4, 0, [0, 3, 1, 5], [1, 5, 40, 5], 4, 2, D, 16)
    o, lse = check_attention(osc, s)
    assert torch.isneginf(lse).any() and (o[0] == 0).all()
    check_attention(osc, make(2, 3, 7, [0, 0, 2], [1, 3, 4], 4, 2, D, 16))  # they see the prefix alone


def test_attention_one_long_request(osc):
    check_attention(osc, make(3, 1, 0, [2900], [1], 4, 1, 128, 64))
    check_attention(osc, make(4, 1, 2100, [1], [1], 4, 1, 64, 32))
    check_attention(osc, make(5, 2, 1000, [900, 3], [3, 2], 4, 2, 128, 16))


@pytest.mark.parametrize("P", [0, 50])
@pytest.mark.parametrize("B", [257, 600, 1100])
def test_attention_many_requests(osc, B, P):
    """more requests than a workgroup has lanes; idle and empty ones among them, and two long ones"""
    gen = np.random.default_rng(B + P)
    n, kv = gen.integers(0, 3, B), gen.integers(0, 40, B)
    n[B // 3], kv[B // 3] = 150, 170
    n[B - 2], kv[B - 2] = 129, 129
    check_attention(osc, make(B + P, B, P, kv.tolist(), n.tolist(), 2, 1, 64, 16))


def test_attention_most_requests(osc):
    gen = np.random.default_rng(2)
    n, kv = gen.integers(0, 2, 8192), gen.integers(0, 20, 8192)
    n[5000], kv[5000] = 300, 320
    check_attention(osc, make(20, 8192, 18, kv.tolist(), n.tolist(), 1, 1, 64, 16))


@pytest.mark.parametrize("P", [0, 300])
def test_attention_behind_a_wide_table(osc, P):
    """rows of the table that could name 2^28 tokens: the work is then counted in larger units"""
    n = [1] * 290 + [40, 70, 1, 33, 5, 130, 1, 1, 1, 64]
    kv = [(7 * b) % 150 + 1 for b in range(290)] + [60, 70, 1000, 33, 5, 500, 1, 2, 700, 64]
    s = make(21 + P, 300, P, kv, n, 8, 8, 64, 256)
    wide = dict(s, table=torch.zeros((300, 1 << 20), dtype=torch.int32, device=DEV))
    wide["table"][:, :s["table"].shape[1]] = s["table"]
    check_attention(osc, s, got=call(osc, wide))
    check_attention(osc, s)


def test_attention_long_prefix(osc):
    """a prefix in several pieces, packed rows of several tiles that cut requests in two"""
    n = [1, 3, 2, 1, 7] * 8
    kv = [5, 3, 40, 100, 9] * 8
    check_attention(osc, make(11, 40, 9001, kv, n, 8, 1, 64, 64))
    check_attention(osc, make(12, 40, 4097, kv, n, 6, 1, 128, 128))


@pytest.mark.parametrize("D,P", [(128, 6500), (64, 9001)])
def test_attention_few_rows_behind_a_long_prefix(osc, D, P):
    """the rows of all requests in one tile of 32 that walks the prefix"""
    check_attention(osc, make(31, 8, P, [5, 200, 33, 1, 64, 90, 17, 40], [1] * 8, 32, 8, D, 64))
    check_attention(osc, make(32, 7, P, [5, 200, 33, 1, 64, 90, 17], [1, 1, 0, 1, 1, 1, 1], 24, 8, D, 128))


def test_attention_few_long_requests(osc):
    """items of many pieces each: tokens of their own, and a prefix that few rows walk"""
    check_attention(osc, make(33, 5, 0, [5000, 1, 7000, 333, 2600], [1, 1, 1, 2, 1], 16, 8, 128, 32))
    check_attention(osc, make(34, 3, 0, [12000, 9000, 31], [1, 3, 1], 8, 8, 64, 128))
    check_attention(osc, make(35, 2, 15000, [300, 5], [1, 1], 32, 8, 128, 64))


@pytest.mark.parametrize("P", [0, 100])
def test_attention_prompts_in_whole_tiles(osc, P):
    """more tiles than workgroups, short enough that none is cut; single tokens beside them"""
    check_attention(osc, make(36 + P, 16, P, [150] * 16, [150] * 16, 32, 8, 128, 64))
    check_attention(osc, make(37 + P, 18, P, [150, 64, 90] * 6, [150, 1, 83] * 6, 24, 8, 64, 32))


@pytest.mark.parametrize("D,P,Hq,Hkv", [(128, 700, 4, 2), (64, 1300, 6, 1), (128, 4100, 8, 8), (64, 4999, 5, 1)])
def test_attention_packed_rows(osc, D, P, Hq, Hkv):
    """the rows of many requests in tiles of 128 that walk the prefix; idle requests between them, and long ones that walk it themselves"""
    gen = np.random.default_rng(P)
    B = 600 if Hkv == 1 else 300 if Hkv == 2 else 60
    n, kv = np.ones(B, int), gen.integers(1, 90, B)
    n[gen.random(B) < 0.1] = 0
    check_attention(osc, make(33, B, P, kv.tolist(), n.tolist(), Hq, Hkv, D, 32))
    n[5], kv[5] = 9, 12
    n[B // 2], kv[B // 2] = 256 * Hkv // Hq + 3, 300
    check_attention(osc, make(34, B, P, np.maximum(kv, n).tolist(), n.tolist(), Hq, Hkv, D, 16))


def test_attention_prompts(osc):
    check_attention(osc, make(13, 2, 100, [500, 410], [500, 300], 4, 2, 128, 16))
    check_attention(osc, make(14, 3, 0, [333, 1, 700], [333, 1, 200], 5, 1, 64, 32))


@pytest.mark.parametrize("D", [64, 128])
def test_attention_many_rows(osc, D):
    """more rows than are joined one a wavefront: few segments each, and many (a short prefix and a long one)"""
    n = [1] * 150 + [60, 130]
    kv = [b % 37 for b in range(150)] + [75, 200]
    check_attention(osc, make(17, 152, 20, kv, n, 30, 5, D, 16))
    check_attention(osc, make(18, 152, 700, kv, n, 30, 5, D, 16))


def test_attention_many_heads_a_key_head(osc):
    check_attention(osc, make(15, 3, 70, [40, 3, 100], [3, 1, 2], 128, 1, 64, 16))
    check_attention(osc, make(16, 3, 0, [40, 3, 100], [3, 1, 2], 100, 1, 128, 16))


def test_attention_sharp_and_flat(osc):
    """scores up to several hundred, whose maximum rises from tile to tile; and all alike"""
    s = make(6, 3, 70, [100, 37, 200], [1, 2, 1], 8, 2, 128, 32, std=40.0)
    check_attention(osc, s)
    s["scale"] = 1e-4
    check_attention(osc, s)
    s["K"] = torch.where(torch.isnan(s["K"]), s["K"], torch.sort(torch.nan_to_num(s["K"]).abs(), dim=2)[0].to(s["K"].dtype))
    s["Q"] = s["Q"].abs()
    s["scale"] = 0.1
    check_attention(osc, s)


def test_attention_bad_pages_stay_inside(osc):
    """page numbers outside the cache: other rows are right, nothing outside is read"""
    s = make(7, 4, 20, [50, 60, 17, 4], [1, 2, 1, 1], 4, 2, 64, 16)
    good, _ = call(osc, s)
    s["table"][1] = -7
    s["K"], s["V"] = torch.nan_to_num(s["K"]), torch.nan_to_num(s["V"])
    o, _ = call(osc, s)
    rows = [0, 3, 4]
    assert torch.equal(o[rows], good[rows])
    s["kv"][2] = 2 ** 30  # longer than its row of the table can say: limited to it
    o, _ = call(osc, s)
    assert torch.equal(o[[0, 4]], good[[0, 4]])
    s["offs"] = i32([0, 5, 1, 5, 2])  # offsets that fall: nothing outside Q is read or written
    call(osc, s)
    torch.cuda.synchronize()


def test_attention_twice_and_in_pieces(osc):
    """the same bits from call to call, and rows do not depend on a workspace's contents"""
    s = make(8, 20, 300, list(range(3, 203, 10)), [1] * 18 + [40, 9], 8, 2, 128, 16)
    n = osc.osc_prefix_attention_workspace_bytes(s["Q"].shape[0], 20, 8, 2, 128, 300)
    first = check_attention(osc, s)
    for fill in (0, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device=DEV)
        again = call(osc, s, workspace=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_step_in_a_graph_and_on_a_stream(osc):
    """slots, norms with rotation and attention of one step, captured once and replayed on new lengths, each replay against the same
    calls made eagerly; on a stream that is not the default one"""
    B, Hq, Hkv, D, ps, width, P = 6, 8, 2, 128, 16, 8, 50
    g = torch.Generator().manual_seed(1)
    n_pages = 80
    K, V = (torch.randn(n_pages, Hkv, ps, D, generator=g).bfloat16().to(DEV) for _ in range(2))
    prefix = i32([70, 71, 72, 73])
    free, cs = i32(np.arange(60)), osc.osc_rope_table(1e4, D, 400)
    gq = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    T = 16
    x = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g).bfloat16().to(DEV)
    kv, q, n_free = i32([0] * B), i32([0] * B), i32([60])
    ws = torch.empty(osc.osc_prefix_attention_workspace_bytes(T, B, Hq, Hkv, D, P), dtype=torch.uint8, device=DEV)

    def step(table, K, V):
        lens, offs, pos, slots, info = osc.osc_page_slots(kv, q, free, n_free, table, ps, T, P)
        y = osc.osc_qk_norm_rope(x, Hq, Hkv, D, cs, pos, slots, K, V, gq, gq)
        o, lse = osc.osc_prefix_attention(y, Hq, Hkv, D, K, V, prefix, P, table, lens, offs, want_lse=True, workspace=ws)
        return lens, offs, pos, slots, info, y, o, lse
    stream = torch.cuda.Stream()
    table = i32(np.zeros((B, width)))
    with torch.cuda.stream(stream):
        step(table, K, V)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs = step(table, K, V)
        gen = np.random.default_rng(0)
        for k in range(5):
            kv.copy_(i32(gen.integers(0, 60, B)))
            q.copy_(i32(gen.integers(0, 3, B)))
            x.copy_(torch.randn(x.shape, generator=g).bfloat16())
            table.copy_(i32(np.arange(B * width).reshape(B, width) % 20))
            t2, K2, V2 = table.clone(), K.clone(), V.clone()
            graph.replay()
            stream.synchronize()
            got = [o.clone() for o in outs]
            eager = step(t2, K2, V2)
            stream.synchronize()
            m = int(eager[1][-1])
            for i, (a, b) in enumerate(zip(got, eager)):
                a, b = (a[:m], b[:m]) if i >= 6 else (a, b)
                assert torch.equal(a, b), (k, i)
            assert torch.equal(table, t2) and torch.equal(K, K2) and torch.equal(V, V2)


# ways through the attention that differ in where a row's sums are finished
WAYS = [("an item a workgroup", lambda D: make(41, 20, 300, list(range(3, 203, 10)), [1] * 18 + [40, 9], 8, 2, D, 16)),
        ("workgroups' pieces, joined", lambda D: make(42, 6, 0, [900, 40, 1200, 7, 650, 33], [1, 2, 1, 1, 1, 3], 8, 2, D, 32)),
        ("long lines, cut", lambda D: make(43, 5, 0, [5000, 1, 7000, 333, 2600], [1, 1, 1, 2, 1], 16, 8, D, 32)),
        ("wavefronts' pieces, joined", lambda D: make(44, 110, 0, [20 + (37 * b) % 280 for b in range(110)], [1] * 110, 8, 8, D, 64)),
        ("whole tiles of prompts", lambda D: make(45, 3, 0, [150, 1, 290], [150, 1, 190], 4, 1, D, 32)),
        ("packed rows", lambda D: make(46, 120, 1300, [1 + (11 * b) % 60 for b in range(120)], [1] * 120, 8, 8, D, 32)),
        ("packed rows and cut prompts, four rows joined a wavefront", lambda D: make(47, 61, 9000, [1 + (13 * b) % 60 for b in range(60)] + [150], [1] * 60 + [130], 24, 8, D, 64))]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("way", range(len(WAYS)), ids=[w for w, _ in WAYS])
def test_attention_queries_that_are_not_finite(osc, way, D):
    """NaN or infinity in a head of a row of queries: that head's result and lse are NaN whichever way it takes; the others are what they
    were (both within the tolerance above, with the largest |v| for the weighted average, 2^-12 of it for the scores' errors, 2^-10 for those of lse)"""
    s = WAYS[way][1](D)
    T, Hq = s["Q"].shape[0], s["Hq"]
    before, lse_before = call(osc, s)
    offs, kv = s["offs"].cpu().numpy(), s["kv"].cpu().numpy()
    b = np.searchsorted(offs, np.arange(T), side="right") - 1
    sees = s["P"] + kv[b] - (offs[b + 1] - np.arange(T)) + 1
    rows = [t for t in range(T) if sees[t] >= 30]  # keys of either sign, so that an infinite element makes infinite scores of either sign
    bad = torch.zeros((T, Hq), dtype=torch.bool, device=DEV)
    for k, t in enumerate(rows[::max(1, len(rows) // 9)]):
        bad[t, 5 * k % Hq] = True
        s["Q"].view(T, Hq, D)[t, 5 * k % Hq, 29 * k % D] = float("nan") if k % 2 else float("inf")
    assert bad.sum() >= 3
    o, lse = call(osc, s)
    o, before = o.view(T, Hq, D), before.view(T, Hq, D)
    assert torch.isnan(o[bad]).all() and torch.isnan(lse[bad]).all()
    top = torch.nan_to_num(s["V"]).abs().max().double()
    err = (o.double() - before.double()).abs()[~bad]
    assert (err <= 2 * (2.0 ** -8 * before.double().abs()[~bad] + (2.0 ** -8 + 2.0 ** -12) * top)).all()
    assert torch.equal(torch.isinf(lse)[~bad], torch.isinf(lse_before)[~bad])
    assert (torch.nan_to_num(lse - lse_before, 0.0)[~bad].abs() <= 2.0 ** -9).all() and not torch.isnan(lse[~bad]).any()


# ---- the attention's ways, each shown to be taken --------------------------------------------------------------------------

# the plan that the first kernel leaves at the workspace's start
PLAN = ("narrow", "wide", "narrow0", "items0", "wide0", "head", "wide_per", "wide_piece", "a", "b", "cut", "with_wide", "others", "piece", "team", "rows", "tiles", "supers",
        "super", "nbp", "valid", "joins")
SOLO, CUT, TEAM, PIECE1, PIECE2, PIECE3 = -1, 0, 5, 3, 6, 12


def lens(seed, B, lo, hi):
    return np.random.default_rng(seed).integers(lo, hi + 1, B).tolist()


# name: for heads of D channels, (prefix, tokens a request has, rows of it, Hq, Hkv, page size); what the plan has to say; rows joined a wavefront
BRANCHES = {
    "an item a workgroup": (lambda D: (300, list(range(3, 203, 10)), [1] * 18 + [40, 9], 8, 2, 16), dict(piece=SOLO, joins=0, rows=0, wide=0), 1),
    "a wavefront's piece an item, nothing joined": (lambda D: (0, lens(1, 110, 1, 160), [1] * 110, 8, 8, 32), dict(piece=PIECE2, joins=0, wide=0), 1),
    "workgroups' pieces": (lambda D: (0, [900, 40, 1200, 7, 650, 33], [1, 2, 1, 1, 1, 3], 8, 2, 32), dict(piece=TEAM, joins=1, items0=0), 1),
    "wavefronts' pieces of 3": (lambda D: (0, lens(2, 110, 20, 200 if D == 128 else 300), [1] * 110, 8, 8, 64), dict(piece=PIECE1, joins=1, items0=0), 1),
    "wavefronts' pieces of 6": (lambda D: (0, lens(3, 110, 250, 400), [1] * 110, 8, 8, 16), dict(piece=PIECE2, joins=1, items0=0), 1),
    "wavefronts' pieces of 12": (lambda D: (0, lens(4, 70 if D == 128 else 110, 700, 1000), [1] * (70 if D == 128 else 110), 8, 8, 128), dict(piece=PIECE3, joins=1), 1),
    "wavefronts' pieces of 12, four rows joined": (lambda D: (0, lens(4, 70 if D == 128 else 110, 700, 900), [1] * (70 if D == 128 else 110), 64, 8, 128),
                                                   dict(piece=PIECE3, joins=1), 4),
    "lines cut": (lambda D: (0, [5000, 1, 7000, 333, 2600], [1, 1, 1, 2, 1], 16, 8, 32), dict(piece=CUT, joins=1, items0=0, with_wide=0), 1),
    "lines cut beside prompts": (lambda D: (0, [9000, 8000, 7000, 9500, 200], [1, 2, 1, 1, 160], 16, 8, 32), dict(piece=CUT, joins=1, wide_piece=SOLO), 1),
    "one tile behind the prefix, workgroups' pieces": (lambda D: (2000, lens(5, 32, 1, 100), [1] * 32, 8, 8, 64), dict(piece=TEAM, items0=8, rows=32, tiles=0, joins=1), 1),
    "one tile behind the prefix, wavefronts' pieces of 3": (lambda D: (8000 if D == 128 else 15000, lens(6, 32, 1, 60), [1] * 32, 8, 8, 64),
                                                            dict(piece=PIECE1, items0=8, rows=32, tiles=0, joins=1), 1),
    "one tile behind the prefix, wavefronts' pieces of 6": (lambda D: (18000, lens(7, 32, 150, 250), [1] * 32, 8, 8, 64) if D == 128 else
                                                            (27000, lens(7, 32, 300, 350), [1] * 32, 8, 8, 64), dict(piece=PIECE2, items0=8, rows=32, tiles=0, joins=1), 1),
    "one tile behind the prefix, lines cut": (lambda D: (15000 if D == 128 else 21000, [40, 300, 5, 17], [1] * 4, 32, 8, 64),
                                              dict(piece=CUT, items0=8, rows=16, tiles=0, joins=1), 1),
    "packed rows, a tile": (lambda D: (1300, lens(8, 120, 1, 60), [1] * 120, 8, 8, 32), dict(tiles=1, supers=5, rows=120, joins=1), 1),
    "packed rows, two tiles": (lambda D: (3000, lens(9, 200, 1, 60), [1] * 200, 8, 8, 32), dict(tiles=2, supers=10, rows=200, joins=1), 1),
    "packed rows, five tiles, four rows joined": (lambda D: (5000, lens(9, 140, 1, 60), [1] * 140, 32, 8, 32), dict(tiles=5, rows=560, joins=1), 4),
    "packed rows beside long requests": (lambda D: (9000, lens(10, 150, 1, 60) + [300], [1] * 150 + [260], 2, 2, 64),
                                         dict(tiles=2, supers=3, rows=150, wide_piece=CUT, joins=1), 1),
    "packed rows beside long requests, four rows joined": (lambda D: (4200, lens(10, 80, 1, 60) + [150], [1] * 80 + [130], 24, 4, 64),
                                                           dict(tiles=4, supers=2, rows=480, wide_piece=CUT, joins=1), 4),
    "prompts cut": (lambda D: (0, [2100, 900], [70, 61], 4, 1, 64), dict(wide_piece=CUT, narrow=0, rows=0, joins=1), 1),
    "prompts behind a prefix cut": (lambda D: (3000, [300, 300], [70, 90], 4, 1, 64), dict(wide_piece=CUT, narrow=0, rows=0, joins=1), 1),
    "prompts behind a prefix cut, four rows joined": (lambda D: (2000, [300, 300], [70, 75], 32, 8, 64), dict(wide_piece=CUT, narrow=0, rows=0, joins=1), 4),
    "prompts whole": (lambda D: (0, [150, 1, 290], [150, 1, 190], 4, 1, 32), dict(wide_piece=SOLO, wide_per=1, joins=0), 1),
    "prompts whole, two tiles a workgroup": (lambda D: (0, [60] * 110, [40] * 110, 8, 8, 32), dict(wide_piece=SOLO, wide_per=2, joins=0), 4),
}


def check_some(osc, s, got, rows):
    """check_attention at some rows; all of them are finite"""
    pick = torch.as_tensor(rows, device=DEV)
    T, Hq, D, scale = s["Q"].shape[0], s["Hq"], s["D"], s["scale"]
    wo, wl, av, big = (w[rows] for w in ref.prefix_attention(f64(s["Q"]).reshape(T, Hq, D), f64(s["K"]), f64(s["V"]), s["prefix"].cpu().numpy(), s["P"], s["table"].cpu().numpy(),
                                                             s["kv"].cpu().numpy(), s["offs"].cpu().numpy(), scale, rows))
    o, lse = got
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    n = s["P"] + int(s["kv"].max())
    score = scale * (D + 4) * 2.0 ** -24 * big
    err = np.abs(f64(o[pick]).reshape(len(rows), Hq, D) - wo)
    assert (err <= 2.0 ** -8 * np.abs(wo) + (2.0 ** -8 + 2 * score[..., None] + 2.0 ** -18) * av).all(), (err / (av + 1e-30)).max()
    assert (np.abs(f64(lse[pick]) - wl) <= score + 2.0 ** -21 * (np.abs(wl) + scale * big) + (n + 8) * 2.0 ** -24).all()


@pytest.mark.parametrize("D", [128, 64])
@pytest.mark.parametrize("name", BRANCHES)
def test_attention_ways(osc, name, D):
    """each way through the plan: it is the one taken, its results are right, and they are the same bits from run to run and whatever the workspace
    held: all ones (NaN in the segments), zeros, another call's"""
    args, want, together = BRANCHES[name]
    P, kv, n, Hq, Hkv, ps = args(D)
    s = make(len(name), len(kv), P, kv, n, Hq, Hkv, D, ps)
    T = s["Q"].shape[0]
    assert together == (1 if T * Hq <= 4096 else 4)
    ws = torch.full((osc.osc_prefix_attention_workspace_bytes(T, len(kv), Hq, Hkv, D, P),), 255, dtype=torch.uint8, device=DEV)
    first = call(osc, s, workspace=ws)
    plan = dict(zip(PLAN, ws[:4 * len(PLAN)].view(torch.int32).tolist()))
    assert {k: plan[k] for k in want} == want, plan
    assert plan["valid"] == 1 and (plan["wide"] > 0) == (plan["with_wide"] > 0)
    some = 1500000 // (Hq * (P + max(kv)))  # rows that the oracle takes about a second for
    if T <= some:
        check_attention(osc, s, got=first)
    else:
        check_some(osc, s, first, sorted(set(np.random.default_rng(1).integers(0, T, max(some, 6)).tolist()) | {0, T - 1}))
    for fill in (0, None):
        if fill is not None:
            ws.fill_(fill)
        again = call(osc, s, workspace=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (24, 8, 64)])
@pytest.mark.parametrize("n", [2048, 8192])
def test_attention_long_prompts(osc, Hq, Hkv, D, n):
    """a prompt of full length, at rows all over it"""
    s = make(n + D, 1, 0, [n], [n], Hq, Hkv, D, 64)
    check_some(osc, s, call(osc, s), [0, 1, 31, 32, 127, 128, 1000, n // 2 - 1, n // 2, n - 129, n - 2, n - 1])
    s = make(n + D + 1, 3, 300, [n // 2 + 40, 5, 900], [n // 2, 1, 700], Hq, Hkv, D, 32)
    check_some(osc, s, call(osc, s), [0, 255, 256, n // 4, n // 2 - 1, n // 2, n // 2 + 1, n // 2 + 700])


@pytest.mark.parametrize("B", [4, 300])
def test_attention_leaves_other_rows_alone(osc, B):
    """offsets that fall, or that name rows past the end, compute nothing; rows outside those that the offsets name keep what they hold"""
    kv, n = [5 + b % 40 for b in range(B)], [1 + b % 3 for b in range(B)]
    s = make(50 + B, B, 40, kv, n, 4, 2, 64, 16)
    T = s["Q"].shape[0]
    offs = s["offs"].cpu().numpy()
    swapped, high, negative = offs.copy(), offs.copy(), offs.copy()
    swapped[[1, 2]] = swapped[[2, 1]]
    high[-1] = T + 1
    negative[0] = -1
    for bad in (swapped, high, negative, offs[::-1].copy(), np.full_like(offs, 2 ** 31 - 1), np.full_like(offs, -2 ** 31)):
        o, lse = torch.full((T, 256), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((T, 4), 7.0, device=DEV)
        call(osc, dict(s, offs=i32(bad)), out=(o, lse))
        assert (o == 7).all() and (lse == 7).all()
    # the same requests, rows before and behind them
    more = torch.randn(T + 24, 256, device=DEV).bfloat16()
    more[11:11 + T] = s["Q"]
    o, lse = torch.full((T + 24, 256), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((T + 24, 4), 7.0, device=DEV)
    call(osc, dict(s, Q=more, offs=i32(offs + 11)), out=(o, lse))
    for x in (o, lse):
        assert (x[:11] == 7).all() and (x[11 + T:] == 7).all()
    check_attention(osc, s, got=(o[11:11 + T].contiguous(), lse[11:11 + T].contiguous()))
