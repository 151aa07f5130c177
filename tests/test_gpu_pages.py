"""Cached tokens and pages in other hands, on the GPU against their plain forms (oracle/tree.py): whole numbers and copied values, all
equal."""
import numpy as np
import pytest
import torch

from oracle import tree as ref

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


def caches(seed, layers, pages, Hkv, ps, D):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(layers, pages, Hkv, ps, D, generator=g).bfloat16().to(DEV) for _ in range(2)]


# ---- moves --------------------------------------------------------------------------------------------------------------


def check_move(osc, C, src, dst, offs, flat=False):
    want = [c.cpu().float().numpy().copy() for c in C]
    for w in want:
        ref.cache_move(w, src, dst, offs)
    osc.osc_cache_move(*([c[0] for c in C] if flat else C), i32(src), i32(dst), i32(offs))
    for c, w in zip(C, want):
        assert np.array_equal(c.cpu().float().numpy(), w)


@pytest.mark.parametrize("Hkv,D", [(1, 64), (8, 128), (3, 128), (5, 64)])
@pytest.mark.parametrize("ps", [16, 64, 256])
def test_move_towards_the_start(osc, Hkv, D, ps):
    """accepted tokens of trees: a slot is written after it was read, rows of any number, pairs that move nothing among them"""
    gen = np.random.default_rng(Hkv + ps)
    layers, pages = 1 + Hkv % 3, 6 + 2000 // ps
    C = caches(ps, layers, pages, Hkv, ps, D)
    perm = gen.permutation(pages * ps)
    src, dst, offs, at = [], [], [0], 0
    for n in (1, 2, 7, 64, 65, 0, 130, 300, 33):
        own = perm[at:at + n]
        at += n
        keep = np.flatnonzero(gen.random(n) < (1.0 if n == 33 else 0.5))
        src += own[keep].tolist() + [-1] * (n - len(keep))
        dst += own.tolist()
        offs.append(offs[-1] + n)
    check_move(osc, C, src, dst, offs, flat=layers == 1)


def test_move_forms(osc):
    C = caches(1, 1, 4, 2, 16, 64)
    check_move(osc, C, [3, 64, -1, 5, 2 ** 31 - 1], [9, 1, 2, 64, 8], [0, 5])  # slots that no cache has
    check_move(osc, C, [1, 2], [5, 6], [0, 1])                                  # pairs of no group
    K, V = caches(2, 6, 4, 2, 16, 64)
    want = [c.clone() for c in (K, V)]
    osc.osc_cache_move(K[1::2], V[1::2], i32([[1, 2], [3, -1]]), i32([[9, 10], [60, 11]]))  # layers apart, groups by rows
    for w, c in zip(want, (K, V)):
        w = w.view(6, 4, 2, 16, 64)
        for a, b in ((1, 9), (2, 10), (3, 60)):
            w[1::2, b // 16, :, b % 16] = w[1::2, a // 16, :, a % 16]
        assert torch.equal(w, c)
    before = K.clone()
    osc.osc_cache_move(K, V, i32([1, 2]), i32([5, 6]), i32([0, 3]))  # a group that leaves the list
    osc.osc_cache_move(K, V, i32([1, 2]), i32([5, 6]), i32([-1, 2]))
    osc.osc_cache_move(K, V, i32([]), i32([]))
    osc.osc_cache_move(K, V, i32([1, 2]), i32([5, 6]), i32([0]))
    assert torch.equal(K, before)


def test_move_past_32_bits(osc):
    """a layer of more than 2^32 bytes: the last page's tokens to the first, and back"""
    pages = 2 ** 20 + 3
    K = torch.zeros(pages, 2, 16, 128, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    K[-1], V[-1], K[0, 0], V[0, 1] = 3.0, 5.0, 1.0, 2.0
    last = pages * 16 - 1
    osc.osc_cache_move(K, V, i32([last, 3]), i32([7, last - 2]))
    assert (K[0, :, 7] == 3).all() and (V[0, :, 7] == 5).all() and K[-1, :, 13, 0].tolist() == [1, 0] and V[-1, :, 13, 0].tolist() == [0, 2]
    assert (K[1:-1] == 0).all() and (K[0, 0, :7] == 1).all()


# ---- forks --------------------------------------------------------------------------------------------------------------


def check_fork(osc, src, dst, kv, ps, width, n_pool, n_free, seed=0, n_pages=None, table=None):
    gen = np.random.default_rng(seed)
    B = len(kv)
    pages = gen.permutation(n_pool + B * width)
    free = pages[:n_pool]
    table = pages[n_pool:].reshape(B, width) if table is None else table
    n_pages = len(pages) if n_pages is None else n_pages
    refs = gen.integers(0, 3, n_pages)
    want = ref.page_fork(src, dst, kv, table, refs, free, n_free, ps)
    d_kv, d_table, d_refs = i32(kv), i32(table), i32(refs)
    s, d, info = osc.osc_page_fork(i32(src), i32(dst), d_kv, d_table, d_refs, i32(free), i32([n_free]), ps)
    for name, g, w in zip(("lengths", "table", "refs", "from", "to", "info"), (d_kv, d_table, d_refs, s, d, info), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    return want


@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
def test_fork(osc, ps):
    gen = np.random.default_rng(ps)
    for B, N in ((2, 1), (9, 4), (70, 30), (300, 290), (600, 258), (8192, 2500)):
        rows = gen.permutation(B)
        dst, kept = rows[:N], rows[N:]
        kv = gen.integers(0, 4 * ps + 1, B)
        kv[gen.random(B) < 0.2] = 2 * ps  # full pages alone
        src = gen.choice(kept, N)
        check_fork(osc, src, dst, kv, ps, 4, N + 3, N + 3, seed=B)
        check_fork(osc, src, dst, kv, ps, 4, N + 3, max(0, N // 2), seed=B)  # not enough pages for all


def test_fork_refused(osc):
    kv = [40, 0, 0, 17, 0, 33, 16, -4]
    for src, dst in (([0, 0], [1, 1]), ([0, 3], [3, 1]), ([0], [0]), ([-1, 8, 0, 3], [1, 2, -1, 8]), ([0, 3, 5], [1, 0, 2]), ([7], [1]), ([0, 1, 0], [1, 2, 4]),
                     ([2 ** 31 - 1, -2 ** 31, 0], [1, 2, 4])):
        want = check_fork(osc, src, dst, kv, 16, 4, 9, 9)
        assert want[5][2] >= (src != [7])
    assert check_fork(osc, [0], [1], [65, 3], 16, 4, 9, 9)[5][2] == 1  # more tokens than a row has room for
    for n_free in (-3, 0, 1, 2, 99):
        check_fork(osc, [0, 3, 6, 5], [1, 2, 4, 7], kv, 16, 4, 3, n_free)
    check_fork(osc, [], [], kv, 16, 4, 3, 2)
    check_fork(osc, [0, 0], [1, 2], [40, 0, 0], 16, 4, 5, 5, n_pages=3)  # pages that no cache has are entered, not counted, and nothing of them moved
    check_fork(osc, [0], [1], [40, 0], 16, 3, 4, 4, table=np.array([[-1, 2 ** 31 - 1, -9], [1, 1, 1]]))


# ---- pages given back ---------------------------------------------------------------------------------------------------------


def check_free(osc, kv, new, ps, table, n_pages, n_pool, n_free, refs=None, seed=0):
    gen = np.random.default_rng(seed)
    free = gen.integers(0, 10 ** 6, n_pool)
    wr, wf, wi = ref.page_free(kv, new, table, refs, free, n_free, ps, n_pages)
    d_free, d_refs, d_table = i32(free), None if refs is None else i32(refs), i32(table)
    info = osc.osc_page_free(i32(kv), None if new is None else i32(new), d_table, d_free, i32([n_free]), ps, d_refs, n_pages)
    assert info.tolist() == wi.tolist()
    assert np.array_equal(d_free.cpu().numpy(), wf) and np.array_equal(d_table.cpu().numpy(), table)
    if refs is not None:
        assert np.array_equal(d_refs.cpu().numpy(), wr)
    return wi


@pytest.mark.parametrize("ps", [16, 64, 256])
def test_free(osc, ps):
    gen = np.random.default_rng(ps)
    for B in (1, 2, 63, 64, 65, 300, 1023, 1024, 1025, 8192):
        width = 5
        n_pages = B * width + 7
        table = gen.permutation(n_pages)[:B * width].reshape(B, width)
        kv = gen.integers(0, width * ps + 1, B)
        new = np.minimum(kv, gen.integers(0, width * ps + 1, B))
        new[gen.random(B) < 0.3] = 0
        check_free(osc, kv, new, ps, table, n_pages, n_pages + 3, 3)
        check_free(osc, kv, None, ps, table, n_pages, n_pages + 3, 3, refs=gen.integers(0, 2, n_pages))
        check_free(osc, kv, new, ps, table, n_pages, n_pages // 2, 2)  # a list that is too short


def test_free_shared_pages(osc):
    """pages of several rows: the last holder's release frees them, wherever it stands; released once too often they are freed once"""
    gen = np.random.default_rng(4)
    for seed in range(5):
        table = gen.integers(0, 12, (20, 4))
        holders = np.bincount(table.reshape(-1), minlength=12)
        kv = np.full(20, 64)
        check_free(osc, kv, None, 16, table, 12, 40, 0, refs=np.maximum(holders - 1, 0), seed=seed)  # all let go
        check_free(osc, kv, None, 16, table, 12, 40, 0, refs=holders, seed=seed)                      # one holder stays
        check_free(osc, kv, None, 16, table, 12, 40, 5, refs=np.maximum(holders - 4, 0), seed=seed)
        check_free(osc, kv, gen.integers(0, 65, 20), 16, table, 12, 40, 0, refs=gen.integers(0, 4, 12), seed=seed)
        check_free(osc, kv, None, 16, table, 12, 40, 0, seed=seed)                                    # no counts: named several times, entered once


def test_free_forms(osc):
    table = np.arange(12).reshape(3, 4)
    check_free(osc, [64, 64, 64], [64, 70, 200], 16, table, 12, 20, 4)            # nothing goes
    check_free(osc, [-5, 900, 17], [-3, -9, 3], 16, table, 12, 20, 4)             # lengths below 0 and past the row
    check_free(osc, [64, 64, 64], None, 16, np.array([[-1, 99, 2 ** 31 - 1, 3]] * 3), 12, 20, 4)  # pages that no cache has
    check_free(osc, [64, 64, 64], None, 16, table, 5, 20, 4)
    for n_free in (-7, 0, 19, 20, 99):
        check_free(osc, [64, 64, 64], None, 16, table, 12, 20, n_free)
    check_free(osc, [], None, 16, np.zeros((0, 4), int), 12, 20, 3)
    check_free(osc, [5, 5], None, 16, np.zeros((2, 0), int), 12, 20, 3)
    check_free(osc, [5, 5], None, 16, np.zeros((2, 1), int), 0, 20, 3)            # a cache without pages
    check_free(osc, [5, 5], None, 16, np.ones((2, 1), int), 4, 0, 0)              # no list


def test_free_caches_of_many_pages(osc):
    """more pages than a range of bits, pages of all ranges, ends of ranges among them"""
    gen = np.random.default_rng(6)
    for n_pages in (2 ** 19 - 1, 2 ** 19, 2 ** 19 + 1, 3 * 2 ** 19 + 40):
        edge = [p for r in range(4) for p in (r * 2 ** 19 - 1, r * 2 ** 19, r * 2 ** 19 + 1) if 0 <= p < n_pages] + [n_pages - 1, n_pages - 32, n_pages]
        table = np.concatenate([edge, gen.integers(0, n_pages, 4000 - len(edge))]).reshape(400, 10)
        refs = np.zeros(n_pages, int)
        refs[gen.integers(0, n_pages, n_pages // 3)] = 1
        check_free(osc, np.full(400, 160), None, 16, table, n_pages, 5000, 11, refs=refs)
        check_free(osc, np.full(400, 160), None, 16, table, n_pages, 5000, 11)


def test_deal_fork_free(osc):
    """a search over continuations, step by step: rows dropped and forked, new tokens dealt; every page is in one place, and counts add up"""
    gen = np.random.default_rng(8)
    B, ps, width, n_pages = 12, 16, 9, 80
    free, refs = i32(gen.permutation(n_pages)), i32(np.zeros(n_pages))
    n_free, table = i32([n_pages]), i32(np.full((B, width), -1))
    kv = i32(np.zeros(B))
    for step in range(15):
        q = i32(gen.integers(0, 20 if step == 0 else 4, B))
        kv, _, _, slots, info = osc.osc_page_slots(kv, q, free, n_free, table, ps, int(q.sum()))
        n_free = info[:1].clone()
        rows = gen.permutation(B)
        dst, src = rows[:3], gen.choice(rows[5:], 3)
        new = kv.clone()
        new[torch.as_tensor(dst.copy())] = 0
        info = osc.osc_page_free(kv, new, table, free, n_free, ps, refs)
        from_, to, info = osc.osc_page_fork(i32(src), i32(dst), new, table, refs, free, info[:1], ps)
        assert info[2].item() == 0 and info[0].item() >= 0
        kv, n_free = new.clone(), info[:1].clone()
        lens, t, holders = kv.tolist(), table.tolist(), np.zeros(n_pages, int)
        for b in range(B):
            for j in range(-(-lens[b] // ps)):
                holders[t[b][j]] += 1
                if lens[b] % ps and j == lens[b] // ps:
                    assert refs[t[b][j]].item() == 0  # what is written next is nobody else's
        assert np.array_equal(np.maximum(holders - 1, 0), refs.cpu().numpy())
        listed = free[:n_free.item()].tolist()
        assert len(set(listed)) == len(listed) and all(holders[p] == 0 for p in listed) and len(listed) == (holders == 0).sum()


def test_most_requests_and_many_pages(osc):
    gen = np.random.default_rng(9)
    n_pages, B = 2 ** 19 + 77, 8192
    table = gen.integers(0, n_pages, (B, 9))
    refs = gen.integers(0, 2, n_pages)
    check_free(osc, gen.integers(0, 145, B), gen.integers(0, 60, B), 16, table, n_pages, 90000, 40, refs=refs)
    rows = gen.permutation(B)
    check_fork(osc, gen.choice(rows[4096:], 4096), rows[:4096], gen.integers(0, 65, B), 16, 4, 5000, 4100)


def test_shorter_than_the_fork(osc):
    """a request that goes back behind the token where it was forked: a fork of its own, and the other holder's tokens stay what they were"""
    ps, width, n_pages = 16, 4, 20
    K, V = caches(3, 2, n_pages, 2, ps, 64)
    table, free, refs = i32(np.full((3, width), -1)), i32(np.arange(n_pages)[::-1].copy()), i32(np.zeros(n_pages))
    kv, _, _, slots, info = osc.osc_page_slots(i32([0, 0, 0]), i32([40, 0, 0]), free, i32([n_pages]), table, ps, 40)
    tokens = lambda C, row, n: C[:, table[row].long()[torch.arange(n, device=DEV) // ps], :, torch.arange(n, device=DEV) % ps].clone()
    first = [tokens(C, 0, 40) for C in (K, V)]
    a, b, info = osc.osc_page_fork(i32([0]), i32([1]), kv, table, refs, free, info[:1].clone(), ps)
    osc.osc_cache_move(K, V, a, b)
    assert kv.tolist() == [40, 40, 0] and refs[table[1, 1].long()].item() == 1
    # row 1 back to 20 tokens, inside a page that row 0 holds too: into row 2
    kv[1] = 20
    a, b, info = osc.osc_page_fork(i32([1]), i32([2]), kv, table, refs, free, info[:1].clone(), ps)
    osc.osc_cache_move(K, V, a, b)
    kv[1] = 40
    new = kv.clone()
    new[1] = 0
    info = osc.osc_page_free(kv, new, table, free, info[:1].clone(), ps, refs)
    assert info[1:].tolist() == [1, 2, 0] and new.tolist() == [40, 0, 20]
    kv, _, _, slots, info = osc.osc_page_slots(new, i32([0, 0, 20]), free, info[:1].clone(), table, ps, 20)
    assert (slots >= 0).all()
    for C in (K, V):
        C[:, slots.long() // ps, :, slots.long() % ps] = 9.0
    for C, was in zip((K, V), first):
        assert torch.equal(tokens(C, 0, 40), was)
        now = tokens(C, 2, 40)  # [tokens, layers, heads, D]
        assert torch.equal(now[:20], was[:20]) and (now[20:] == 9).all()
    held = {p for r, n in ((0, 3), (2, 3)) for p in table[r, :n].tolist()}
    listed = free[:info[0].item()].tolist()
    assert len(set(listed)) == len(listed) and not held & set(listed) and len(held) + len(listed) == n_pages


def test_refused_forks_after_pages_were_given_back(osc):
    """rows are dropped, the list has pages for some of the forks alone: the others are empty requests, and every page is in one place"""
    ps, width, B, n_pages = 16, 3, 8, 26
    table, free, refs = i32(np.full((B, width), -1)), i32(np.arange(n_pages)), i32(np.zeros(n_pages))
    kv, _, _, _, info = osc.osc_page_slots(i32([0] * B), i32([40] * B), free, i32([n_pages]), table, ps, 40 * B)
    assert info[0].item() == 2
    n_free, new = info[:1].clone(), kv.clone()
    new[4:] = 0
    info = osc.osc_page_free(kv, new, table, free, n_free, ps, refs)
    few = info[:1].clone() - 12  # as if others had taken twelve since
    _, _, forked = osc.osc_page_fork(i32([0, 0, 1, 3]), i32([4, 5, 6, 7]), new, table, refs, free, few, ps)
    assert few.item() == 2 and forked.tolist() == [0, 2, 2, 4] and new.tolist() == [40, 40, 40, 40, 40, 40, 0, 0]
    holders = np.zeros(n_pages, int)
    for b, n in enumerate(new.tolist()):
        for j in range(-(-n // ps)):
            holders[table[b, j].item()] += 1
    assert np.array_equal(np.maximum(holders - 1, 0), refs.cpu().numpy())
    gone = osc.osc_page_free(new, None, table, free, i32([0]), ps, refs)
    assert gone.tolist() == [14, 14, 4, 0] and (refs == 0).all() and sorted(free[:14].tolist()) == sorted(np.flatnonzero(holders))


@pytest.mark.parametrize("B", [400, 1024, 1025, 3000])
@pytest.mark.parametrize("n_pages", [2 ** 19 + 1, 3 * 2 ** 19 + 40])
def test_free_few_pages_a_request_of_many_ranges(osc, n_pages, B):
    """no request lets more than eight pages go: pages of all ranges of bits, ends of ranges, the same page several times, pages that no cache has; one request
    a thread and several"""
    gen = np.random.default_rng(B)
    edge = [p for r in range(4) for p in (r * 2 ** 19 - 1, r * 2 ** 19, r * 2 ** 19 + 1, r * 2 ** 19 + 31, r * 2 ** 19 + 32) if 0 <= p < n_pages] + [n_pages - 1, n_pages - 32]
    table = gen.integers(0, n_pages, (B, 9))
    flat = table.reshape(-1)
    flat[gen.permutation(flat.size)[:8 * len(edge)]] = np.tile(edge, 8)
    flat[gen.permutation(flat.size)[:90]] = np.tile([-1, n_pages, n_pages + 5, 2 ** 31 - 1, -2 ** 31, -2 ** 19], 15)
    kv = gen.integers(0, 145, B)
    new = np.maximum(kv - gen.integers(0, 129, B), 0)   # up to nine pages held, eight of them let go at most
    keep = -(-new // 16)
    assert (-(-kv // 16) - keep).max() == 8
    refs = np.zeros(n_pages, int)
    refs[gen.integers(0, n_pages, n_pages // 3)] = 1
    refs[edge] = gen.integers(0, 9, len(edge))
    wi = check_free(osc, kv, new, 16, table, n_pages, 30000, 11, refs=refs)
    assert wi[1] > B and wi[2] > 0 and wi[3] > 0
    check_free(osc, kv, new, 16, table, n_pages, 30000, 11)
    check_free(osc, kv, new, 16, table, n_pages, B, 11, refs=refs)   # a list that is too short
    check_free(osc, np.minimum(kv, 128), None, 16, table, n_pages, 30000, 0, refs=refs)
