"""What the operators of speculative decoding refuse, on the host and before any launch; and their plain forms against hand-made
cases.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_12782_amd as osc
from oracle import tree as ref

NULL, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -4, -5
P = 1 << 16  # stands for a device pointer: refused calls never look at it


def rc(fn, **kw):
    name, defaults = fn
    args = dict(defaults, **kw)
    assert set(args) == set(defaults), set(args) - set(defaults)
    return getattr(osc.lib(), name)(*args.values())


MASK = ("osc_tree_mask", dict(par=P, offs=2 * P, kv=3 * P, B=4, T=8, base=0, words=1, mask=4 * P, ldm=1, pos=5 * P, stream=None))
ATTN = ("osc_tree_attention", dict(Q=P, T=4, Hq=8, Hkv=2, D=128, ldq=1024, K=P, V=P, n_pages=9, ps=16, pp=P, P=40, table=P, ldt=5, kv=P, offs=P, B=4,
                                   mask=P, words=1, ldm=1, scale=0.1, O=P, ldo=1024, lse=None, ws=P, nb=0, stream=None))
ACCEPT = ("osc_tree_accept", dict(par=P, tok=2 * P, ch=3 * P, ldc=1, offs=4 * P, kv=5 * P, slots=6 * P, B=4, T=8, path=7 * P, n=8 * P, nxt=9 * P, kv_out=10 * P,
                                  src=11 * P, stream=None))
MOVE = ("osc_cache_move", dict(K=P, V=2 * P, layers=1, stride=0, n_pages=9, Hkv=2, ps=16, D=128, src=3 * P, dst=4 * P, offs=5 * P, N=2, T=8, stream=None))
FORK = ("osc_page_fork", dict(src=P, dst=2 * P, N=3, B=4, ps=16, kv=3 * P, table=4 * P, ldt=5, refs=5 * P, n_pages=9, free=6 * P, n_pool=9, n_free=7 * P, from_=8 * P,
                              to=9 * P, info=10 * P, stream=None))
FREE = ("osc_page_free", dict(kv=P, new=2 * P, B=4, ps=16, table=3 * P, ldt=5, refs=4 * P, n_pages=9, free=5 * P, n_pool=9, n_free=6 * P, info=7 * P, stream=None))
LOGP = ("osc_token_logprobs", dict(x=P, dtype=0, T=4, V=50000, ldl=50000, scale=1.0, tok=P, n=1, k=5, lp=P, ids=P, top=P, lse=P, ent=P, ws=P, nb=1 << 30, stream=None))


@pytest.mark.parametrize("code,change", [
    (SHAPE, dict(B=-1)), (SHAPE, dict(T=-1)), (UNSUPPORTED, dict(B=8193)), (UNSUPPORTED, dict(T=2 ** 31)), (SHAPE, dict(base=-1)), (UNSUPPORTED, dict(words=0)),
    (UNSUPPORTED, dict(words=9, ldm=9)), (SHAPE, dict(words=2)), (SHAPE, dict(ldm=2 ** 31)), (NULL, dict(par=None)), (NULL, dict(offs=None)), (NULL, dict(kv=None)),
    (NULL, dict(mask=None)), (NULL, dict(pos=None)), (UNSUPPORTED, dict(mask=4 * P + 4)), (UNSUPPORTED, dict(pos=4 * P + 60)), (UNSUPPORTED, dict(pos=P + 28)),
    (UNSUPPORTED, dict(mask=2 * P + 16)), (UNSUPPORTED, dict(pos=3 * P)), (0, dict(T=0, par=None))])
def test_mask_refusals(code, change):
    assert rc(MASK, **change) == code


@pytest.mark.parametrize("code,change", [
    (SHAPE, dict(Hq=7)), (UNSUPPORTED, dict(D=80)), (UNSUPPORTED, dict(ps=20)), (SHAPE, dict(T=-1)), (SHAPE, dict(B=-1)), (UNSUPPORTED, dict(B=8193)),
    (UNSUPPORTED, dict(P=2 ** 30)), (SHAPE, dict(ldq=1016)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=float("nan"))), (NULL, dict(Q=None)), (NULL, dict(O=None)),
    (NULL, dict(kv=None)), (NULL, dict(offs=None)), (NULL, dict(ws=None)), (NULL, dict(table=None)), (NULL, dict(pp=None)), (NULL, dict(K=None)), (UNSUPPORTED, dict(Q=P + 2)),
    (UNSUPPORTED, dict(O=P + 8)), (UNSUPPORTED, dict(ws=P + 16)), (UNSUPPORTED, dict(words=0)), (UNSUPPORTED, dict(words=9, ldm=9)), (SHAPE, dict(words=3, ldm=2)),
    (NULL, dict(mask=None)), (UNSUPPORTED, dict(mask=P + 4)), (WORKSPACE, dict()), (0, dict(T=0, Q=None, mask=None)), (0, dict(B=0, kv=None))])
def test_attention_refusals(code, change):
    assert rc(ATTN, **change) == code
    if code < 0:
        assert osc.osc_last_error().startswith("osc_tree_attention")


@pytest.mark.parametrize("code,change", [
    (SHAPE, dict(B=-1)), (SHAPE, dict(T=-1)), (UNSUPPORTED, dict(B=8193)), (UNSUPPORTED, dict(T=2 ** 31)), (SHAPE, dict(ldc=0)), (SHAPE, dict(ldc=2 ** 31)),
    *[(NULL, {k: None}) for k in ("par", "tok", "ch", "offs", "kv", "slots", "path", "n", "nxt", "kv_out", "src")], (UNSUPPORTED, dict(src=6 * P)),
    (UNSUPPORTED, dict(kv_out=5 * P)), (UNSUPPORTED, dict(path=3 * P + 8)), (UNSUPPORTED, dict(ch=7 * P - 4 * 50, ldc=8)), (0, dict(B=0, T=0, par=None, path=None))])
def test_accept_refusals(code, change):
    assert rc(ACCEPT, **change) == code


@pytest.mark.parametrize("code,change", [
    (SHAPE, dict(Hkv=0)), (UNSUPPORTED, dict(D=96)), (UNSUPPORTED, dict(D=0)), (UNSUPPORTED, dict(ps=24)), (SHAPE, dict(n_pages=-1)), (SHAPE, dict(n_pages=2 ** 27)),
    (UNSUPPORTED, dict(K=P + 8)), (UNSUPPORTED, dict(V=P + 8)), (SHAPE, dict(layers=-1)), (SHAPE, dict(N=-1)), (SHAPE, dict(T=-1)), (SHAPE, dict(layers=2, stride=9 * 2 * 16 * 128 - 8)),
    (UNSUPPORTED, dict(layers=2, stride=9 * 2 * 16 * 128 + 4)), (UNSUPPORTED, dict(layers=65536, stride=9 * 2 * 16 * 128)), (UNSUPPORTED, dict(T=2 ** 31)),
    (SHAPE, dict(offs=None, N=3)), *[(NULL, {k: None}) for k in ("K", "V", "src", "dst")], (0, dict(N=0, src=None)), (0, dict(T=0, src=None)), (0, dict(layers=0, K=None)),
    (0, dict(n_pages=0, K=None, V=None))])
def test_move_refusals(code, change):
    assert rc(MOVE, **change) == code


@pytest.mark.parametrize("code,change", [
    (UNSUPPORTED, dict(ps=8)), (UNSUPPORTED, dict(ps=512)), (SHAPE, dict(N=-1)), (SHAPE, dict(B=-1)), (SHAPE, dict(ldt=-1)), (SHAPE, dict(n_pages=-1)), (SHAPE, dict(n_pool=-1)),
    (UNSUPPORTED, dict(N=8193)), (UNSUPPORTED, dict(B=8193)), (UNSUPPORTED, dict(n_pages=2 ** 27)), (UNSUPPORTED, dict(n_pool=2 ** 31)), (UNSUPPORTED, dict(ldt=2 ** 29)),
    *[(NULL, {k: None}) for k in ("src", "dst", "kv", "table", "refs", "free", "n_free", "from_", "to", "info")], (UNSUPPORTED, dict(n_free=10 * P)), (UNSUPPORTED, dict(to=8 * P + 4)),
    (UNSUPPORTED, dict(src=3 * P + 12)), (UNSUPPORTED, dict(free=4 * P + 40))])
def test_fork_refusals(code, change):
    assert rc(FORK, **change) == code


@pytest.mark.parametrize("code,change", [
    (UNSUPPORTED, dict(ps=17)), (SHAPE, dict(B=-1)), (SHAPE, dict(ldt=-1)), (SHAPE, dict(n_pages=-1)), (SHAPE, dict(n_pool=-1)), (UNSUPPORTED, dict(B=8193)),
    (UNSUPPORTED, dict(n_pages=2 ** 31)), (UNSUPPORTED, dict(n_pool=2 ** 31)), (UNSUPPORTED, dict(ldt=2 ** 29)), *[(NULL, {k: None}) for k in ("kv", "table", "free", "n_free", "info")],
    (UNSUPPORTED, dict(n_free=7 * P + 4)), (UNSUPPORTED, dict(refs=5 * P)), (UNSUPPORTED, dict(free=3 * P + 8)), (UNSUPPORTED, dict(free=2 * P))])
def test_free_refusals(code, change):
    assert rc(FREE, **change) == code


@pytest.mark.parametrize("code,change", [
    (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(dtype=-1)), (SHAPE, dict(T=-1)), (SHAPE, dict(V=0)), (SHAPE, dict(ldl=49999)), (SHAPE, dict(n=-1)), (SHAPE, dict(k=-1)),
    (SHAPE, dict(V=4, k=5)), (UNSUPPORTED, dict(k=65)), (UNSUPPORTED, dict(T=2 ** 31)), (UNSUPPORTED, dict(V=2 ** 31, ldl=2 ** 31)), (SHAPE, dict(scale=0.0)),
    (SHAPE, dict(scale=-1.0)), (SHAPE, dict(scale=float("nan"))), (SHAPE, dict(scale=float("inf"))), *[(NULL, {k: None}) for k in ("x", "tok", "lp", "ids", "top", "ws")],
    (UNSUPPORTED, dict(x=P + 2)), (UNSUPPORTED, dict(x=P + 1, dtype=1)), (UNSUPPORTED, dict(ws=P + 16)), (WORKSPACE, dict(nb=64)), (0, dict(T=0, x=None))])
def test_logprobs_refusals(code, change):
    assert rc(LOGP, **change) == code


def test_workspace_sizes():
    size = osc.osc_tree_attention_workspace_bytes
    assert size(4, 4, 8, 2, 128, 40) > 0
    for bad in ((-1, 4, 8, 2, 128, 40), (4, -1, 8, 2, 128, 40), (4, 4, 8, 3, 128, 40), (4, 4, 8, 2, 96, 40), (4, 4, 8, 2, 128, -1), (4, 8193, 8, 2, 128, 0)):
        assert size(*bad) == 0
    size = osc.osc_token_logprobs_workspace_bytes
    assert size(1, 131072, 8) > 0 and size(100000, 131072, 8) == 0 and size(0, 100, 0) == 0
    for bad in ((-1, 10, 0), (1, 0, 0), (1, 131072, 65), (1, 5, 6), (1, 131072, -1)):
        assert size(*bad) == 0


def test_binding_refuses_wrong_tensors():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    h = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    f = lambda *s: torch.zeros(s)

    def refused(fn, good, *bad):
        for k, v in bad:
            with pytest.raises(AssertionError):
                fn(**dict(good, **{k: v}))
    good = dict(parents=i(5), q_offsets=i(3), kv_lens=i(2), out=(torch.zeros(5, 1, dtype=torch.int64), i(5)))
    refused(osc.osc_tree_mask, good, ("parents", i(5).long()), ("q_offsets", i(2)), ("kv_lens", i(4)), ("out", (torch.zeros(5, 2, dtype=torch.int64), i(5))), ("words", 0),
            ("out", (i(5, 1), i(5))), ("out", (torch.zeros(5, 1, dtype=torch.int64), i(4))), ("parents", i(10)[::2]), ("kv_lens", i(2)))  # the last: not on a GPU
    good = dict(Q=h(5, 512), Hq=4, Hkv=1, D=128, Kc=h(4, 1, 16, 128), Vc=h(4, 1, 16, 128), prefix_pages=i(2), prefix_len=20, block_table=i(3, 4), kv_lens=i(3),
                q_offsets=i(4), mask=torch.zeros(5, 1, dtype=torch.int64), workspace=torch.zeros(1 << 20, dtype=torch.uint8), out=(h(5, 512), None))
    refused(osc.osc_tree_attention, good, ("mask", i(5, 1)), ("mask", torch.zeros(4, 1, dtype=torch.int64)), ("mask", torch.zeros(5, dtype=torch.int64)),
            ("mask", torch.zeros(5, 4, dtype=torch.int64)[:, ::2]), ("Q", h(5, 504)), ("Q", h(5, 512).half()), ("kv_lens", i(2)), ("out", (h(5, 256), None)))
    good = dict(parents=i(5), tokens=i(5), choices=i(5), q_offsets=i(3), kv_lens=i(2), slots=i(5), out=(i(5), i(2), i(2), i(2), i(5)))
    refused(osc.osc_tree_accept, good, ("tokens", i(4)), ("choices", i(5, 1)), ("choices", i(5).long()), ("choices", i(4)), ("slots", i(4)), ("q_offsets", i(2)),
            ("out", (i(5), i(2), i(2), i(2), i(4))), ("kv_lens", i(2)))
    good = dict(Kc=h(2, 1, 16, 64), Vc=h(2, 1, 16, 64), src_slots=i(4), dst_slots=i(4))
    refused(osc.osc_cache_move, good, ("Kc", h(2, 1, 16, 64).float()), ("Vc", h(3, 1, 16, 64)), ("Kc", h(2, 16, 1, 64).transpose(1, 2)), ("dst_slots", i(3)), ("src_slots", i(4).long()),
            ("Vc", h(1, 2, 1, 16, 64)), ("offsets", i(0)), ("offsets", i(3).long()), ("Kc", h(2, 1, 16, 64).half()), ("src_slots", i(4)))
    good = dict(src=i(2), dst=i(2), kv_lens=i(3), block_table=i(3, 4), refs=i(9), free_pages=i(9), n_free=i(1), page_size=16, out=(i(2, 16), i(2, 16), i(4)))
    refused(osc.osc_page_fork, good, ("dst", i(1)), ("src", i(2).long()), ("block_table", i(2, 4)), ("block_table", i(4, 3).t()), ("refs", i(9).short()), ("n_free", i(0)),
            ("out", (i(2, 8), i(2, 16), i(4))), ("page_size", 0), ("kv_lens", i(3)))
    good = dict(kv_lens=i(3), new_lens=i(3), block_table=i(3, 4), free_pages=i(9), n_free=i(1), page_size=16, refs=i(9), out=i(4))
    refused(osc.osc_page_free, good, ("new_lens", i(2)), ("block_table", i(3, 4).long()), ("free_pages", i(9).short()), ("n_pages", 10), ("out", i(3)), ("kv_lens", i(3)))
    good = dict(logits=f(4, 100), tokens=i(4), top_k=3, out=(f(4), i(4, 3), f(4, 3), f(4), f(4)), workspace=torch.zeros(64, dtype=torch.uint8))
    refused(osc.osc_token_logprobs, good, ("logits", f(4, 100).half()), ("logits", f(100)), ("logits", f(100, 4).t()), ("tokens", i(3)), ("tokens", i(4).long()),
            ("out", (f(4), i(4, 2), f(4, 3), f(4), f(4))), ("out", (f(3), i(4, 3), f(4, 3), f(4), f(4))), ("top_k", -1), ("tokens", i(4)))


def test_plain_trees_by_hand():
    par = [-1, 0, 0, 2, 1, -1, 0]
    mask, pos = ref.tree_mask(par, [0, 5, 7], [25, 4], 8, 1, 100)
    assert mask[:, 0].tolist() == [1, 3, 5, 13, 19, 1, 3, 0] and pos.tolist() == [120, 121, 121, 122, 122, 102, 103, -1]
    long, at = ref.tree_mask(np.arange(65) - 1, [0, 65], [65], 65, 1)
    assert not long.any() and at.tolist() == list(range(65))
    path, count, following, lens, src = ref.tree_accept(par, [9, 4, 5, 6, 7, 1, 2], [5, 0, 6, 8, 0, 3, 0], [0, 5, 7], [25, 4], [10, 11, 12, 13, 14, 30, 31], 8)
    assert path.tolist() == [0, 2, 3, -1, -1, 0, -1, -1] and src.tolist() == [10, 12, 13, -1, -1, 30, -1, -1]
    assert count.tolist() == [3, 1] and following.tolist() == [8, 3] and lens.tolist() == [23, 3]


def test_plain_tree_attention_of_a_chain_is_causal():
    from oracle import attention
    rng = np.random.default_rng(1)
    K, V = rng.standard_normal((5, 1, 16, 64)), rng.standard_normal((5, 1, 16, 64))
    q = rng.standard_normal((3, 2, 64))
    mask, _ = ref.tree_mask([-1, 0, 1], [0, 3], [18], 3, 1)
    a = ref.tree_attention(q, K, V, [4, 2], 20, np.array([[3, 0]]), [18], [0, 3], mask, 0.2)
    b = attention.prefix_attention(q, K, V, [4, 2], 20, np.array([[3, 0]]), [18], [0, 3], 0.2)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_plain_pages_by_hand():
    kv, table, refs, src, dst, info = ref.page_fork([0, 0, 3], [1, 2, 1], [20, 0, 0, 5], [[7, 8], [0, 0], [0, 0], [9, 0]], [0] * 12, [1, 2, 3], 3, 16)
    assert kv.tolist() == [20, 20, 20, 5] and table.tolist() == [[7, 8], [7, 3], [7, 2], [9, 0]] and refs[7] == 2 and info.tolist() == [1, 2, 1, 2]
    assert src[0, :4].tolist() == [128, 129, 130, 131] and dst[1, :5].tolist() == [32, 33, 34, 35, -1] and (src[2] == -1).all()
    refs, free, info = ref.page_free(kv, [0, 0, 16, 5], table, refs, [1, 2, 3, 0, 0, 0], 1, 16, 12)
    assert free.tolist() == [1, 2, 3, 8, 0, 0] and info.tolist() == [4, 3, 2, 0] and refs[7] == 0


def test_plain_logprobs_against_torch():
    x = torch.randn(4, 50, dtype=torch.float64, generator=torch.Generator().manual_seed(0))
    lp, ids, top, lse, ent = ref.token_logprobs(x.numpy(), np.array([[1], [2], [49], [50]]), 5, 1.5)
    want = torch.log_softmax(1.5 * x, 1)
    assert np.allclose(lp[:3, 0], want[[0, 1, 2], [1, 2, 49]]) and lp[3, 0] == 0 and np.allclose(lse, torch.logsumexp(1.5 * x, 1))
    assert np.allclose(top, want.topk(5).values) and np.array_equal(ids, want.topk(5).indices) and np.allclose(ent, -(want.exp() * want).sum(1))


def test_extents_past_32_bits():
    """overlap checks hold for pitches whose last element lies past 2^32 bytes, and past 2^64"""
    assert rc(ACCEPT, ch=8 * P, ldc=2 ** 31 - 1, T=2 ** 31 - 1, par=P) == UNSUPPORTED   # whatever is behind it is inside
    assert rc(MASK, T=2 ** 31 - 1, ldm=2 ** 30 - 1, pos=2 ** 40) == UNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(lp=100 * P), dict(lse=100 * P + 799996), dict(lp=P), dict(ids=P - 76), dict(top=3 * P + 76), dict(ent=5 * P + 12), dict(ws=2 * P), dict(tok=7 * P + 1532),
    dict(dtype=1, T=3, V=1, ldl=2 ** 62, k=0, n=0, tok=None, lse=2 ** 50)])
def test_logprobs_outputs_apart(change):
    good = dict(x=100 * P, tok=P, lp=2 * P, ids=3 * P, top=4 * P, lse=5 * P, ent=6 * P, ws=7 * P)
    assert rc(LOGP, **dict(good, **change)) == UNSUPPORTED and "overlaps" in osc.osc_last_error()


@pytest.mark.parametrize("change", [dict(N=2 ** 26, T=2 ** 26, Hkv=1, offs=None), dict(N=2 ** 23, T=2 ** 23, Hkv=8, offs=None)])
def test_move_of_too_many_groups(change):
    assert rc(MOVE, **change) == UNSUPPORTED


LAUNCHES = r"""
/* the runtime's calls around a launch: what was to be launched is written down, nothing runs */
#include <stddef.h>
typedef struct { unsigned x, y, z; } dim;
int launches = 0;
unsigned grids[64][3], blocks[64];
static dim grid, block;
int __hipPushCallConfiguration(dim g, dim b, size_t lds, void *stream) { grid = g, block = b; return 0; }
int __hipPopCallConfiguration(dim *g, dim *b, size_t *lds, void **stream) { *g = grid, *b = block, *lds = 0, *stream = NULL; return 0; }
int hipLaunchKernel(const void *f, dim g, dim b, void **args, size_t lds, void *stream) {
    if (launches < 64) grids[launches][0] = g.x, grids[launches][1] = g.y, grids[launches][2] = g.z, blocks[launches] = b.x;
    ++launches;
    return 0;
}
int hipGetLastError(void) { return 0; }
"""
LAUNCHES_CHILD = r"""
import ctypes as C, sys
stub = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
lib = C.CDLL(sys.argv[2])
lib.osc_token_logprobs_workspace_bytes.restype = C.c_size_t
vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
P = 1 << 62
for T, V, k in ((1 << 23, 131072, 5), ((1 << 23) + 1, 131072, 5), ((1 << 23) + 60, 40000, 3), ((2 << 23) + 128, 200000, 0)):
    need = lib.osc_token_logprobs_workspace_bytes(i64(T), i64(V), i32(k))
    at = C.c_int.in_dll(stub, "launches")
    at.value = 0
    rc = lib.osc_token_logprobs(vp(1 << 20), 1, i64(T), i64(V), i64(V), C.c_float(1.0), None, i32(0), i32(k), None, vp(P), vp(P + (1 << 58)), vp(P + (2 << 58)), None,
                                None, C.c_size_t(0), None)
    grids = (C.c_uint * 3 * 64).in_dll(stub, "grids")
    blocks = (C.c_uint * 64).in_dll(stub, "blocks")
    print(T, need, rc, [(grids[i][0], grids[i][1], blocks[i]) for i in range(at.value)])
"""


def test_rows_of_several_launches_need_no_workspace(tmp_path):
    """a call's rows past 2^23 are launched as the others are: whole rows, no second kernel, nothing of a workspace that the call does not ask for"""
    import ast
    import subprocess
    import sys
    src, so = tmp_path / "launches.c", tmp_path / "launches.so"
    src.write_text(LAUNCHES)
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", str(src), "-o", str(so)], check=True)
    p = subprocess.run([sys.executable, "-c", LAUNCHES_CHILD, str(so), osc.lib_path()], capture_output=True, text=True, timeout=120)
    assert p.returncode == 0, p.stderr[-2000:]
    lines = [l.split(maxsplit=3) for l in p.stdout.splitlines()]
    assert len(lines) == 4
    for T, need, code, launched in lines:
        rows = [min(2 ** 23, int(T) - r) for r in range(0, int(T), 2 ** 23)]
        assert need == "0" and code == "0" and ast.literal_eval(launched) == [(n, 1, 256) for n in rows], (T, launched)


@pytest.mark.parametrize("Hkv,N", [(1, 2 ** 26 - 3), (1, 2 ** 26 - 2), (1, 2 ** 26 - 1), (3, (2 ** 26 - 1) // 3), (2, 2 ** 25 - 1)])
def test_move_of_the_first_groups_that_are_too_many(Hkv, N):
    """four heads of groups a workgroup of 256, rounded up: from 2^26 - 3 on a launch would have 2^32 threads"""
    assert N * Hkv > 2 ** 26 - 4 and rc(MOVE, N=N, T=N, Hkv=Hkv, offs=None) == UNSUPPORTED


def test_move_of_as_many_groups_as_there_may_be():
    assert rc(MOVE, N=2 ** 26 - 4, T=0, Hkv=1, offs=None) == 0
