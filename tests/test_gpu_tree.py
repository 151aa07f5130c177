"""Trees of drafted tokens on the GPU against their plain forms in 64 bits (oracle/tree.py): bits and positions, attention of the
trees' rows, accepted paths.

Tolerances of the attention: those of the attention behind a shared prefix (bf16 results rounded once, 2^-8 of the value; weights rounded
to bf16 before the second product, 2^-8 of the weighted average of |v|; scores are sums of D products)."""
import numpy as np
import pytest
import torch

from oracle import tree as ref
from test_gpu_attention import f64, i32, make

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def osc():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_12782_amd as m
    m.lib()
    return m


def draft(gen, n, how):
    """parents of a tree: a chain, a star, any earlier row, or a forest with rows that continue nothing"""
    i = np.arange(n)
    if how == "chain":
        return i - 1
    if how == "star":
        return np.where(i > 0, 0, -1)
    p = np.where(gen.random(n) < 0.5, i - 1, (gen.random(n) * i).astype(int))
    p[:1] = -1
    if how == "forest":
        p[gen.random(n) < 0.2] = -1
        p[gen.random(n) < 0.05] = n + 5     # no earlier row: none
        p[gen.random(n) < 0.05] = -2 ** 31
        p = np.where(gen.random(n) < 0.05, i, p)
    return p


HOWS = ["any", "chain", "star", "forest"]


def trees(seed, counts):
    gen = np.random.default_rng(seed)
    return np.concatenate([draft(gen, n, HOWS[(seed + b) % 4]) for b, n in enumerate(counts)] or [np.zeros(0, int)]).astype(int)


def words_of(mask):
    return mask.cpu().numpy().view(np.uint64)


# ---- bits and positions ------------------------------------------------------------------------------------------------


def check_mask(osc, counts, kv, words, base=0, before=0, behind=0, seed=0):
    offs = before + np.concatenate([[0], np.cumsum(counts)]).astype(int)
    T = int(offs[-1]) + behind
    par = np.full(T, 7)
    par[before:offs[-1]] = trees(seed, counts)
    mask, pos = osc.osc_tree_mask(i32(par), i32(offs), i32(kv), words, base)
    wm, wp = ref.tree_mask(par, offs, kv, T, words, base)
    assert np.array_equal(words_of(mask), wm) and np.array_equal(pos.cpu().numpy(), wp)
    return par, offs


@pytest.mark.parametrize("words", [1, 2, 3, 8])
def test_mask(osc, words):
    top = 64 * words
    counts = [1, 2, 63, 64, top, top - 1, top + 1, 0, 5, 300, top // 2 + 3, 1, 0]
    for seed in range(4):
        check_mask(osc, counts, [n + 11 * i for i, n in enumerate(counts)], words, base=3 * seed, seed=seed)
    check_mask(osc, counts, [n // 2 for n in counts], words)           # fewer tokens than rows: positions stop at -1
    check_mask(osc, counts, counts, words, before=3, behind=700, seed=2)  # rows of no request
    check_mask(osc, [-n for n in range(0)], [], words, behind=5)


def test_mask_strides_and_many_requests(osc):
    gen = np.random.default_rng(1)
    counts = gen.integers(0, 9, 8192)
    check_mask(osc, counts, counts + gen.integers(0, 99, 8192), 1, base=10, behind=33)
    par, offs = check_mask(osc, [70, 3], [90, 3], 2)
    wide = torch.full((73, 5), 77, dtype=torch.int64, device=DEV)
    pos = torch.full((73,), 77, dtype=torch.int32, device=DEV)
    osc.osc_tree_mask(i32(par), i32(offs), i32([90, 3]), 2, 0, out=(wide[:, 1:3], pos))
    assert np.array_equal(words_of(wide[:, 1:3].contiguous()), ref.tree_mask(par, offs, [90, 3], 73, 2)[0]) and (wide[:, 3:] == 77).all() and (wide[:, 0] == 77).all()


def test_mask_of_offsets_that_fall(osc):
    """a request whose rows are not there is left out; nothing outside the arrays is touched"""
    mask, pos = (torch.full(s, 77, dtype=t, device=DEV) for s, t in (((6, 1), torch.int64), ((6,), torch.int32)))
    osc.osc_tree_mask(i32([-1, 0, 1, -1, 0, 1]), i32([0, 3, 2, 9]), i32([3, 3, 3]), 1, 0, out=(mask, pos))
    assert mask[:3, 0].tolist() == [1, 3, 7] and pos[:3].tolist() == [0, 1, 2]


# ---- attention -----------------------------------------------------------------------------------------------------------


def tree_of(seed, s, counts, words):
    offs = s["offs"].cpu().numpy()
    mask, _ = ref.tree_mask(trees(seed, counts), offs, s["kv"].cpu().numpy(), int(offs[-1]), words)
    return torch.from_numpy(mask.view(np.int64)).to(DEV)


def call(osc, s, mask, **kw):
    return osc.osc_tree_attention(s["Q"], s["Hq"], s["Hkv"], s["D"], s["K"], s["V"], s["prefix"], s["P"], s["table"], s["kv"], s["offs"], mask, s["scale"],
                                  want_lse=True, **kw)


def check(osc, s, mask, got=None):
    o, lse = call(osc, s, mask) if got is None else got
    T, D, scale = s["Q"].shape[0], s["D"], s["scale"]
    wo, wl, av, big = ref.tree_attention(f64(s["Q"]).reshape(T, s["Hq"], D), f64(s["K"]), f64(s["V"]), s["prefix"].cpu().numpy(), s["P"], s["table"].cpu().numpy(),
                                         s["kv"].cpu().numpy(), s["offs"].cpu().numpy(), words_of(mask.contiguous()), scale)
    n = s["P"] + int(s["kv"].max())
    score = scale * (D + 4) * 2.0 ** -24 * big
    err = np.abs(f64(o).reshape(T, s["Hq"], D) - wo)
    assert (err <= 2.0 ** -8 * np.abs(wo) + (2.0 ** -8 + 2 * score[..., None] + 2.0 ** -18) * av).all(), (err / (av + 1e-30)).max()
    empty = np.isinf(wl)
    assert np.array_equal(np.isneginf(f64(lse)), empty)
    tol = score + 2.0 ** -21 * (np.abs(np.where(empty, 0, wl)) + scale * big) + (n + 8) * 2.0 ** -24
    assert (np.abs(np.where(empty, 0, f64(lse)) - np.where(empty, 0, wl)) <= tol).all()
    return o, lse


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (8, 2, 128), (6, 2, 64), (3, 3, 64), (12, 1, 128), (40, 8, 64), (48, 1, 64)])
@pytest.mark.parametrize("P", [0, 1, 33, 250])
def test_attention(osc, Hq, Hkv, D, P):
    """every alignment of a tree's first token to the tiles of 32 and 64; chains, stars, forests"""
    counts = [1, 2, 7, 16, 31, 32, 33, 64, 5, 1, 40, 0]
    kv = [1, 33, 70, 16, 95, 96, 129, 64, 100, 32, 163, 9]
    s = make(P + Hq, len(kv), P, kv, counts, Hq, Hkv, D, 16 << ((Hq + P) % 5))
    check(osc, s, tree_of(P, s, counts, 1))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("words", [1, 2, 3, 8])
def test_attention_wide_trees(osc, words, D):
    """trees of every number of words, and pieces of prompts beside them, which have no tree"""
    top = 64 * words
    counts = [min(top, 150), 64 * words + 1, 3, min(top, 129), top - 1 if top < 200 else 65]
    kv = [c + e for c, e in zip(counts, (37, 0, 90, 64, 11))]
    for P in (0, 20):
        s = make(words + P, len(kv), P, kv, counts, 4, 2, D, 32)
        check(osc, s, tree_of(words, s, counts, words))


def test_attention_any_mask(osc):
    """masks that are no tree's: none of the new tokens, all, every second, not oneself, later rows' bits set (ignored)"""
    counts, kv = [40, 20, 9, 70, 3], [40, 85, 9, 131, 3]
    for P in (0, 18):
        s = make(9, len(kv), P, kv, counts, 8, 2, 128, 16)
        T = sum(counts)
        gen = np.random.default_rng(P)
        for m in (np.zeros((T, 2)), np.full((T, 2), -1), np.full((T, 2), 0x5555555555555555), gen.integers(-2 ** 63, 2 ** 63 - 1, (T, 2))):
            o, lse = check(osc, s, torch.from_numpy(m.astype(np.int64)).to(DEV))
            if not m.any() and P == 0:
                assert torch.isneginf(lse[0]).all() and (o[0] == 0).all()  # nothing is cached before this request's tokens
    check(osc, s, torch.full((T, 2), -1, device=DEV))


def test_attention_strided_mask_rows(osc):
    counts, kv = [33, 70], [60, 99]
    s = make(4, 2, 5, kv, counts, 4, 1, 64, 16)
    mask = tree_of(3, s, counts, 2)
    wide = torch.full((103, 6), -1, dtype=torch.int64, device=DEV)
    wide[:, 2:4] = mask
    a, b = call(osc, s, mask), call(osc, s, wide[:, 2:4])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("P", [0, 700, 3000])
def test_attention_batches(osc, P):
    """lines that are cut, packed rows, items a workgroup and a wavefront"""
    gen = np.random.default_rng(P)
    for B, most, long in ((1, 12, 2500), (40, 12, 300), (9, 70, 900), (3, 128, 1500)):
        counts = gen.integers(1, most + 1, B).tolist()
        kv = [n + int(gen.integers(0, long)) for n in counts]
        s = make(B + P, B, P, kv, counts, 4, 1, 128 if B != 9 else 64, 64)
        mask = tree_of(B, s, counts, 2)
        o, lse = check(osc, s, mask)
        for _ in range(2):
            again = call(osc, s, mask)
            assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_attention_bad_tables_and_offsets(osc):
    """page numbers that no cache has are read as page 0; offsets out of order compute nothing; short lengths of refused requests"""
    counts, kv = [20, 9], [30, 40]
    s = make(2, 2, 0, kv, counts, 4, 2, 64, 16)
    mask = tree_of(0, s, counts, 1)
    t = dict(s, table=torch.full_like(s["table"], -7), K=torch.nan_to_num(s["K"]), V=torch.nan_to_num(s["V"]))
    zero = dict(t, table=torch.zeros_like(s["table"]))
    assert torch.equal(call(osc, t, mask)[0], call(osc, zero, mask)[0])
    out = torch.full((29, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    osc.osc_tree_attention(s["Q"], 4, 2, 64, s["K"], s["V"], s["prefix"], 0, s["table"], s["kv"], i32([0, 25, 20]), mask, out=(out, None))
    assert (out == 7).all()
    short = make(3, 2, 0, [30, 4], counts, 4, 2, 64, 16)  # fewer tokens than rows: the first ones see nothing
    check(osc, short, tree_of(0, short, counts, 1))


def test_attention_workspace_contents_do_not_matter(osc):
    counts, kv = [30, 64, 9], [2000, 900, 700]
    s = make(6, 3, 900, kv, counts, 8, 2, 128, 32)
    mask = tree_of(1, s, counts, 1)
    n = osc.osc_tree_attention_workspace_bytes(103, 3, 8, 2, 128, 900)
    got = [call(osc, s, mask, workspace=torch.full((n,), f, dtype=torch.uint8, device=DEV)) for f in (0, 255, 127)]
    for g in got[1:]:
        assert torch.equal(g[0], got[0][0]) and torch.equal(g[1], got[0][1])


# ---- accepted paths ---------------------------------------------------------------------------------------------------------


def check_accept(osc, counts, kv, par, tokens, choices, slots, before=0, behind=0, ldc=1):
    offs = before + np.concatenate([[0], np.cumsum(counts)]).astype(int)
    T = int(offs[-1]) + behind
    pad = lambda x: np.concatenate([np.full(before, 3), x, np.full(T - before - len(x), 3)]).astype(int)
    par, tokens, choices, slots = pad(par), pad(tokens), pad(choices), pad(slots)
    wide = torch.full((max(T, 1), ldc), -9, dtype=torch.int32, device=DEV)
    wide[:T, 0] = i32(choices)
    got = osc.osc_tree_accept(i32(par), i32(tokens), wide[:T, 0], i32(offs), i32(kv), i32(slots))
    want = ref.tree_accept(par, tokens, choices, offs, kv, slots, T)
    for name, g, w in zip(("path", "count", "next", "lengths", "source"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name
    return want


@pytest.mark.parametrize("ldc", [1, 8])
def test_accept(osc, ldc):
    gen = np.random.default_rng(ldc)
    longest = 0
    for seed in range(6):
        counts = [1, 2, 8, 63, 64, 65, 0, 130, 200, 7, 512]
        par = trees(seed, counts)
        T = len(par)
        few = 3 if seed % 2 else 2  # tokens that agree often, and with several children
        tokens, choices = gen.integers(0, few, T), gen.integers(0, few, T)
        tokens[gen.random(T) < 0.1 * (seed % 3)] = -1
        want = check_accept(osc, counts, [n + 5 for n in counts], par, tokens, choices, gen.integers(0, 10 ** 6, T), before=seed, behind=100 * (seed % 2), ldc=ldc)
        longest = max(longest, want[1].max())
    assert longest > 3  # some paths are paths


def test_accept_chains_branches_prompts(osc):
    n = 200
    chain, zeros = np.arange(n) - 1, np.zeros(n, int)
    assert check_accept(osc, [n], [n], chain, zeros, zeros, np.arange(n))[1][0] == n           # all of a chain
    for stop in (0, 1, 62, 63, 64, 65, 127, 198):                                                # the chain breaks behind this row
        choices = zeros.copy()
        choices[stop] = 5
        want = check_accept(osc, [n], [n + 9], chain, zeros, choices, np.arange(n))
        assert want[1][0] == stop + 1 and want[2][0] == 5 and want[3][0] == 9 + stop + 1
    assert check_accept(osc, [n], [n], chain, zeros - 1, np.arange(n) + 7, np.arange(n))[2][0] == n + 6  # a prompt's tokens
    far = np.full(n, -1)
    far[150], far[199] = 0, 150                                                                  # children in other blocks of 64
    assert check_accept(osc, [n], [n], far, zeros, zeros, np.arange(n))[1][0] == 3
    twice = np.array([-1, 0, 0, 0, 2, 1])                                                        # equal drafts: the lowest row
    assert check_accept(osc, [6], [6], twice, [0, 4, 4, 4, 0, 0], [4, 9, 0, 0, 0, 0], np.arange(6))[0].tolist()[:2] == [0, 1]


def test_accept_refused_and_idle_requests(osc):
    counts, kv = [3, 0, 4, 2], [10, 8, 0, 2]
    par = np.array([-1, 0, 1, -1, 0, 1, 2, -1, 0])
    slots = np.array([5, 6, 7, -1, -1, -1, -1, 3, 4])
    want = check_accept(osc, counts, kv, par, np.zeros(9, int), np.zeros(9, int), slots)
    assert want[1].tolist() == [3, 0, 0, 2] and want[3].tolist() == [10, 8, 0, 2] and want[2].tolist() == [0, -1, -1, 0]
    gen = np.random.default_rng(0)
    counts = gen.integers(0, 6, 8192)
    check_accept(osc, counts, counts + 3, trees(1, counts), gen.integers(0, 2, counts.sum()), gen.integers(0, 2, counts.sum()), gen.integers(0, 99, counts.sum()), behind=70)
    lens = i32([9, 4])
    out = osc.osc_tree_accept(i32([-1, 0]), i32([0, 0]), i32([0, 0]), i32([0, 9, 2]), lens, i32([1, 2]))  # offsets that leave the step: no rows
    assert out[1].tolist() == [0, 0] and out[3].tolist() == [9, 4]


@pytest.mark.parametrize("D", [64, 128])
def test_attention_queries_that_are_not_finite(osc, D):
    """NaN or infinity in one head of one row: that head is NaN, others are what they were; a head that sees nothing stays zero"""
    for P, counts, kv in ((0, [9, 40, 3], [30, 300, 3]), (400, [9, 40, 3], [30, 300, 3])):
        s = make(7 + P, 3, P, kv, counts, 4, 2, D, 16)
        mask = tree_of(0, s, counts, 1)
        mask[49] = 0  # the last request's first row sees no new token
        before, lse0 = check(osc, s, mask)
        for row, bad in ((3, float("nan")), (20, float("inf")), (49, float("nan"))):
            t = dict(s, Q=s["Q"].clone())
            t["Q"][row, 5] = bad
            o, lse = call(osc, t, mask)
            hit = torch.zeros(52, 4, dtype=torch.bool, device=DEV)
            hit[row, 0] = P > 0 or row != 49
            nan = torch.isnan(o.view(52, 4, D))
            assert torch.equal(torch.isnan(lse), hit) and torch.equal(nan.all(-1), hit) and torch.equal(nan.any(-1), hit)
            keep = ~hit
            assert torch.equal(o.view(52, 4, D)[keep], before.view(52, 4, D)[keep]) and torch.equal(lse[keep], lse0[keep])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("own", [20, 900])
def test_attention_of_trees_of_33_to_64_rows_behind_a_prefix(osc, own, D):
    """their requests walk the prefix themselves where they have many tokens of their own, and packed otherwise"""
    counts = [9, 10, 16, 12, 8, 17, 33]
    kv = [c + own + 5 * i for i, c in enumerate(counts)]
    s = make(own, len(kv), 700, kv, counts, 8, 2, D, 32)
    mask = tree_of(1, s, counts, 1)
    check(osc, s, mask)


def test_attention_most_requests(osc):
    gen = np.random.default_rng(2)
    counts, kv = gen.integers(0, 3, 8192), gen.integers(0, 20, 8192)
    counts[5000], kv[5000] = 70, 120
    kv = np.maximum(kv, counts)
    s = make(20, 8192, 18, kv.tolist(), counts.tolist(), 1, 1, 64, 16)
    check(osc, s, tree_of(0, s, counts.tolist(), 2))


def test_two_calls_at_once(osc):
    """two streams, a workspace each, neither the default one: each as if alone"""
    sets, counts = [], ([7] * 12, [40, 3, 12] * 4)
    for i, c in enumerate(counts):
        s = make(40 + i, 12, 300 * i, [k + 700 for k in c], c, 8, 2, 128, 16)
        mask = tree_of(i, s, c, 1)
        o, lse = call(osc, s, mask)
        n = osc.osc_tree_attention_workspace_bytes(sum(c), 12, 8, 2, 128, 300 * i)
        sets.append((s, mask, o.clone(), lse.clone(), torch.empty(n, dtype=torch.uint8, device=DEV), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = ([], [])
    for _ in range(10):
        for i, (s, mask, _, _, ws, stream) in enumerate(sets):
            with torch.cuda.stream(stream):
                got[i].append(call(osc, s, mask, workspace=ws))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, sets[i][2]) and torch.equal(lse, sets[i][3])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [0, 300])
@pytest.mark.parametrize("what,bad", [("V", float("nan")), ("V", float("inf")), ("K", float("nan")), ("V", float("-inf"))])
def test_attention_of_drafts_that_are_not_finite(osc, what, bad, P, D):
    """rows that see such a draft are NaN in its head, all others what they were: requests of few rows, of more, of two tiles, a piece of a prompt"""
    counts, kv = [9, 40, 60, 20, 100, 16], [30, 300, 461, 21, 130, 16]
    s = make(11 + P, 6, P, kv, counts, 4, 2, D, 16)
    mask = tree_of(0, s, counts, 1)
    before, lse0 = check(osc, s, mask)
    bits, offs = words_of(mask)[:, 0], np.concatenate([[0], np.cumsum(counts)])
    for b, draft, h in ((0, 3, 1), (1, 17, 0), (2, 40, 1), (3, 19, 0), (4, 70, 1), (5, 0, 0), (2, 59, 0)):
        j = kv[b] - counts[b] + draft
        page = int(s["table"][b, j // 16])
        T = s[what].clone()
        T[page, h, j % 16, 5 if what == "V" and b % 2 else slice(None)] = bad
        o, lse = call(osc, dict(s, **{what: T}), mask)
        sees = np.zeros((sum(counts), 4), bool)
        for i in range(counts[b]):
            r = offs[b] + i
            sees[r, 2 * h:2 * h + 2] = i >= draft if counts[b] > 64 else bits[r] >> np.uint64(draft) & np.uint64(1)
        assert sees.any()
        sees = torch.from_numpy(sees).to(DEV)
        got, was = o.view(-1, 4, D), before.view(-1, 4, D)
        hit = torch.isnan(got)  # a prompt's later rows see a value in its channel alone
        assert torch.equal(hit[:, :, 5] if what == "V" else hit.all(-1), sees) and torch.equal(hit.any(-1), sees)
        assert torch.equal(got[~sees], was[~sees])
        if what == "V":
            assert torch.equal(lse, lse0)
        else:
            assert torch.equal(torch.isnan(lse), sees) and torch.equal(lse[~sees], lse0[~sees])


def test_attention_of_drafts_that_are_not_finite_in_long_requests(osc):
    """the same where the new tokens are in several blocks, words and pieces of a request"""
    counts, kv = [97, 5, 300], [5000, 40, 320]
    s = make(3, 3, 0, kv, counts, 6, 2, 64, 32)
    mask = tree_of(1, s, counts, 2)
    before, lse0 = check(osc, s, mask)
    bits = words_of(mask)
    for b, draft in ((0, 2), (0, 63), (0, 64), (0, 96), (2, 0), (2, 150), (2, 299)):
        j, at = kv[b] - counts[b] + draft, [0, 97, 102][b]
        V = s["V"].clone()
        V[int(s["table"][b, j // 32]), 1, j % 32] = float("nan")
        o, lse = call(osc, dict(s, V=V), mask)
        sees = np.zeros((402, 6), bool)
        for i in range(counts[b]):
            sees[at + i, 3:] = i >= draft if b == 2 else bits[at + i, draft // 64] >> np.uint64(draft % 64) & np.uint64(1)
        sees = torch.from_numpy(sees).to(DEV)
        got, was = o.view(-1, 6, 64), before.view(-1, 6, 64)
        assert torch.equal(torch.isnan(got).all(-1), sees) and torch.equal(torch.isnan(got).any(-1), sees)
        assert torch.equal(got[~sees], was[~sees]) and torch.equal(lse, lse0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [0, 300])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf")])
def test_attention_of_drafts_with_an_infinite_key(osc, bad, P, D):
    """an infinite key acts through its scores: a row whose score is infinity is NaN, one whose score is -infinity is as if it did not see the token, and
    a row that sees nothing else is as one that sees nothing; requests of few rows, of more, of two tiles, a piece of a prompt"""
    counts, kv = [9, 40, 60, 20, 100, 16], [30, 300, 461, 21, 130, 16]
    s = make(23 + P, 6, P, kv, counts, 4, 2, D, 16)
    mask = tree_of(0, s, counts, 1)
    bits, offs = words_of(mask)[:, 0], np.concatenate([[0], np.cumsum(counts)])
    q = f64(s["Q"]).reshape(-1, 4, D)
    plain = [f64(s["V"]), s["prefix"].cpu().numpy(), P, s["table"].cpu().numpy(), s["kv"].cpu().numpy(), s["offs"].cpu().numpy(), words_of(mask), s["scale"]]
    big = ref.tree_attention(q, f64(s["K"]), *plain)[3]
    kinds = set()
    for b, draft, h in ((0, 3, 1), (1, 17, 0), (2, 40, 1), (3, 19, 0), (4, 70, 1), (5, 0, 0), (2, 59, 0)):
        j, c = kv[b] - counts[b] + draft, 7 + b
        K = s["K"].clone()
        K[int(s["table"][b, j // 16]), h, j % 16, c] = bad
        o, lse = call(osc, dict(s, K=K), mask)
        sees = np.zeros((sum(counts), 4), bool)
        for i in range(counts[b]):
            r = offs[b] + i
            sees[r, 2 * h:2 * h + 2] = i >= draft if counts[b] > 64 else bits[r] >> np.uint64(draft) & np.uint64(1)
        score = np.where(sees, np.where(q[:, :, c] == 0, np.nan, np.sign(q[:, :, c]) * bad), 0.0)
        got, z = f64(o).reshape(-1, 4, D), f64(lse)
        out = sees & (np.isposinf(score) | np.isnan(score))
        assert np.array_equal(np.isnan(got).all(-1), out) and np.array_equal(np.isnan(got).any(-1), out) and np.array_equal(np.isnan(z), out)
        with np.errstate(invalid="ignore"):
            wo, wl, av, _ = ref.tree_attention(q, f64(K), *plain)
        alone = sees & np.isneginf(score) & np.isnan(wl)  # of its only token a row has a score of -infinity
        assert (got[alone] == 0).all() and np.isneginf(z[alone]).all()
        # check()'s tolerances, with the scores of finite keys.  Rows that do not see the token are held to them too, not to equal bits: a wavefront's rows
        # move the base of their sums together, and an infinite score moves it
        keep = ~out & ~alone
        err = (s["scale"] * (D + 4) * 2.0 ** -24 * big)[keep]
        assert (np.abs(got - wo)[keep] <= 2.0 ** -8 * np.abs(wo[keep]) + (2.0 ** -8 + 2 * err[:, None] + 2.0 ** -18) * av[keep]).all()
        empty = np.isneginf(wl[keep])
        assert np.array_equal(np.isneginf(z[keep]), empty)
        tol = err + 2.0 ** -21 * (np.abs(np.where(empty, 0, wl[keep])) + s["scale"] * big[keep]) + (P + max(kv) + 8) * 2.0 ** -24
        assert (np.abs(np.where(empty, 0, z[keep]) - np.where(empty, 0, wl[keep])) <= tol).all()
        kinds |= {n for n, m in (("out", out), ("left", sees & keep)) if m.any()}
    assert kinds == {"out", "left"}
