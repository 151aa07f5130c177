"""What the operators around the paged cache refuse, on the host and before any launch; and their 64-bit plain forms against
hand-made cases.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2604_12782_amd as osc
from oracle import attention as ref

NULL, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -4, -5
P = 4096  # stands for a device pointer: refused calls never look at it


def rc(fn, **kw):
    names, defaults = fn
    args = dict(defaults, **kw)
    assert set(args) == set(defaults), set(args) - set(defaults)
    sections = args.get("sections")
    if isinstance(sections, list):
        args["sections"] = (C.c_int32 * len(sections))(*sections)
    return getattr(osc.lib(), names)(*args.values())


SLOTS = ("osc_page_slots", dict(kv=P, q=2 * P, B=4, ps=16, free=3 * P, n_pool=9, n_free=4 * P, table=5 * P, ldt=6, base=0, T=8, kv_out=6 * P, offs=7 * P,
                                pos=8 * P, slots=9 * P, info=10 * P, stream=None))
ROPE = ("osc_qk_norm_rope", dict(x=P, T=4, Hq=8, Hkv=2, D=128, ldx=1536, gq=P, gk=P, eps=1e-6, cs=P, n_pos=10, rot=128, style=0, pos=P, ldpos=4,
                                 sections=None, n_axes=1, slots=P, y=P, ldq=1024, K=P, V=P, n_pages=3, ps=16, stream=None))
ATTN = ("osc_prefix_attention", dict(Q=P, T=4, Hq=8, Hkv=2, D=128, ldq=1024, K=P, V=P, n_pages=9, ps=16, pp=P, P=40, table=P, ldt=5, kv=P, offs=P, B=4,
                                     scale=0.1, O=P, ldo=1024, lse=None, ws=P, nb=0, stream=None))
TABLE = ("osc_rope_table", dict(base=1e4, rot=64, n_pos=8, out=P, stream=None))


@pytest.mark.parametrize("code,change", [
    (UNSUPPORTED, dict(ps=0)), (UNSUPPORTED, dict(ps=8)), (UNSUPPORTED, dict(ps=48)), (UNSUPPORTED, dict(ps=512)), (SHAPE, dict(B=-1)), (SHAPE, dict(T=-1)),
    (SHAPE, dict(ldt=-1)), (SHAPE, dict(n_pool=-1)), (SHAPE, dict(base=-1)), (UNSUPPORTED, dict(B=8193)), (UNSUPPORTED, dict(T=2 ** 31)), (NULL, dict(kv=None)),
    (NULL, dict(q=None)), (NULL, dict(n_free=None)), (NULL, dict(kv_out=None)), (NULL, dict(offs=None)), (NULL, dict(info=None)), (NULL, dict(free=None)),
    (NULL, dict(table=None)), (NULL, dict(slots=None)), (NULL, dict(pos=None)), (UNSUPPORTED, dict(kv_out=P)), (UNSUPPORTED, dict(kv_out=P + 12)),
    (UNSUPPORTED, dict(n_free=10 * P)), (0, dict(B=0, kv=None, q=None))])
def test_slots_refusals(code, change):
    assert rc(SLOTS, **change) == code


@pytest.mark.parametrize("code,change", [
    (SHAPE, dict(Hq=7)), (SHAPE, dict(Hq=0)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(T=-1)), (UNSUPPORTED, dict(D=96)), (UNSUPPORTED, dict(D=0)),
    (UNSUPPORTED, dict(Hq=1024, Hkv=1024, ldx=2 ** 20, ldq=2 ** 20)), (UNSUPPORTED, dict(T=2 ** 29, ldpos=2 ** 30)), (NULL, dict(K=None)), (NULL, dict(V=None)),
    (UNSUPPORTED, dict(ps=24)), (SHAPE, dict(n_pages=-1)), (SHAPE, dict(n_pages=2 ** 27)), (UNSUPPORTED, dict(K=P + 8)), (SHAPE, dict(rot=136)),
    (SHAPE, dict(rot=60)), (SHAPE, dict(rot=-8)), (UNSUPPORTED, dict(style=2)), (UNSUPPORTED, dict(n_axes=0)), (UNSUPPORTED, dict(n_axes=4, sections=[64, 0, 0, 0])),
    (NULL, dict(n_axes=2)), (SHAPE, dict(n_axes=2, sections=[32, 31])), (SHAPE, dict(n_axes=2, sections=[65, -1])), (SHAPE, dict(n_axes=2, sections=[32, 32], ldpos=3)),
    (SHAPE, dict(ldx=1528)), (SHAPE, dict(ldq=1016)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=float("nan"))), (SHAPE, dict(n_pos=-1)), (NULL, dict(x=None)),
    (NULL, dict(y=None)), (NULL, dict(pos=None)), (NULL, dict(cs=None)), (NULL, dict(slots=None)), (UNSUPPORTED, dict(x=P + 2)), (UNSUPPORTED, dict(ldx=1540)),
    (UNSUPPORTED, dict(ldq=1028)), (UNSUPPORTED, dict(gq=P + 4)), (UNSUPPORTED, dict(cs=P + 4)), (0, dict(T=0, x=None))])
def test_rope_refusals(code, change):
    assert rc(ROPE, **change) == code


@pytest.mark.parametrize("code,change", [
    (SHAPE, dict(Hq=7)), (UNSUPPORTED, dict(D=80)), (UNSUPPORTED, dict(ps=20)), (SHAPE, dict(T=-1)), (SHAPE, dict(B=-1)), (SHAPE, dict(ldt=-1)), (SHAPE, dict(P=-1)),
    (UNSUPPORTED, dict(B=8193)), (UNSUPPORTED, dict(P=2 ** 30)), (SHAPE, dict(ldq=1016)), (SHAPE, dict(ldo=1016)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=-1.0)),
    (UNSUPPORTED, dict(Hq=129, Hkv=1, D=64, ldq=129 * 64, ldo=129 * 64)), (SHAPE, dict(scale=float("nan"))), (SHAPE, dict(scale=float("inf"))), (NULL, dict(Q=None)), (NULL, dict(O=None)), (NULL, dict(kv=None)), (NULL, dict(offs=None)),
    (NULL, dict(ws=None)), (NULL, dict(table=None)), (NULL, dict(pp=None)), (NULL, dict(K=None)), (NULL, dict(V=None)), (NULL, dict(n_pages=0)),
    (UNSUPPORTED, dict(Q=P + 2)), (UNSUPPORTED, dict(ldq=1028)), (UNSUPPORTED, dict(O=P + 8)), (UNSUPPORTED, dict(ldo=1028)), (UNSUPPORTED, dict(ws=P + 16)),
    (UNSUPPORTED, dict(K=P + 4)), (WORKSPACE, dict()), (0, dict(T=0, Q=None)), (0, dict(B=0, kv=None))])
def test_attention_refusals(code, change):
    assert rc(ATTN, **change) == code


@pytest.mark.parametrize("code,change", [(SHAPE, dict(rot=0)), (SHAPE, dict(rot=60)), (SHAPE, dict(n_pos=-1)), (SHAPE, dict(base=0.0)), (SHAPE, dict(base=float("nan"))),
                                         (UNSUPPORTED, dict(n_pos=2 ** 31)), (NULL, dict(out=None)), (0, dict(n_pos=0, out=None))])
def test_rope_table_refusals(code, change):
    assert rc(TABLE, **change) == code


def test_workspace_size():
    size = osc.osc_prefix_attention_workspace_bytes
    assert size(4, 4, 8, 2, 128, 40) > 0
    for bad in ((-1, 4, 8, 2, 128, 40), (4, -1, 8, 2, 128, 40), (4, 4, 8, 3, 128, 40), (4, 4, 8, 2, 96, 40), (4, 4, 8, 2, 128, -1), (4, 4, 0, 2, 128, 0)):
        assert size(*bad) == 0


def test_binding_refuses_wrong_tensors():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    h = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    good = dict(kv_lens=i(3), q_lens=i(3), free_pages=i(9), n_free=i(1), block_table=i(3, 4), page_size=16, T=8)
    for k, v in (("kv_lens", i(3).long()), ("q_lens", i(2)), ("q_lens", i(3).long()), ("n_free", i(0)), ("block_table", i(2, 4)), ("block_table", i(12)),
                 ("block_table", i(4, 3).t()), ("free_pages", i(9).short())):
        with pytest.raises(AssertionError):
            osc.osc_page_slots(**dict(good, **{k: v}))
    with pytest.raises(AssertionError):
        osc.osc_page_slots(**good, out=(i(3), i(3), i(8), i(8), i(4)))
    good = dict(QKV=h(5, 768), Hq=4, Hkv=1, D=128, cos_sin=torch.zeros(9, 128), positions=i(5), slots=i(5), Kc=h(2, 1, 16, 128), Vc=h(2, 1, 16, 128), gamma_q=h(128),
                gamma_k=h(128), out=h(5, 512))
    for k, v in (("QKV", h(5, 760)), ("QKV", torch.zeros(5, 768)), ("cos_sin", torch.zeros(9, 128).double()), ("positions", i(4)), ("positions", i(5).long()),
                 ("positions", i(2, 2, 5)), ("slots", i(4)), ("Kc", h(2, 2, 16, 128)), ("Vc", h(3, 1, 16, 128)), ("Vc", h(2, 1, 32, 128)), ("gamma_q", h(64)),
                 ("out", h(4, 512)), ("out", h(5, 504))):
        with pytest.raises(AssertionError):
            osc.osc_qk_norm_rope(**dict(good, **{k: v}))
    with pytest.raises(AssertionError):
        osc.osc_qk_norm_rope(**dict(good, positions=i(2, 5)), sections=[64])
    with pytest.raises(AssertionError):
        osc.osc_qk_norm_rope(**good, rot=64)
    good = dict(Q=h(5, 512), Hq=4, Hkv=1, D=128, Kc=h(4, 1, 16, 128), Vc=h(4, 1, 16, 128), prefix_pages=i(2), prefix_len=20, block_table=i(3, 4), kv_lens=i(3),
                q_offsets=i(4), workspace=torch.zeros(1 << 20, dtype=torch.uint8), out=(h(5, 512), None))
    for k, v in (("Q", h(5, 504)), ("Kc", h(4, 1, 16, 64)), ("Vc", h(5, 1, 16, 128)), ("prefix_pages", i(1)), ("block_table", i(3, 4).long()), ("block_table", i(3, 8)[:, :4]),
                 ("kv_lens", i(2)), ("q_offsets", i(3)), ("out", (h(5, 256), None)), ("out", (h(5, 512), torch.zeros(5, 3)))):
        with pytest.raises(AssertionError):
            osc.osc_prefix_attention(**dict(good, **{k: v}))


def test_plain_page_slots_by_hand():
    after, offs, pos, slots, info, table = ref.page_slots([3, 16, 0], [2, 1, 17], 16, [7, 8, 9, 5], 3, [[1, -1], [2, -1], [-1, -1]], 21, 100)
    assert after.tolist() == [5, 17, 17] and offs.tolist() == [0, 2, 3, 20]
    assert table.tolist() == [[1, -1], [2, 9], [8, 7]] and info.tolist() == [0, 3, 0, 20]
    assert slots.tolist() == [19, 20, 144, *range(128, 144), 112, -1] and pos.tolist() == [103, 104, 116, *range(100, 117), -1]
    refused = ref.page_slots([3, 16, 0], [2, 1, 17], 16, [7, 8], 2, [[1, -1], [2, -1], [-1, -1]], 20)
    assert refused[0].tolist() == [5, 17, 0] and refused[4].tolist() == [1, 1, 1, 20] and (refused[3][3:] == -1).all()


def test_plain_rotation_keeps_lengths_and_differences():
    """a turned pair keeps its length, and the product of two turned heads depends on the positions' difference alone"""
    rng = np.random.default_rng(0)
    cs = ref.rope_angles(100.0, 8, 50)
    q, k = rng.standard_normal((1, 1, 12)), rng.standard_normal((1, 1, 12))
    for pairs in (False, True):
        turn = lambda x, p: ref.head_rope(x, None, 0.0, cs, np.array([[p]]), [4], 8, pairs)[0]
        a, b = turn(q, 31), turn(k, 20)
        assert np.allclose(np.linalg.norm(a), np.linalg.norm(q)) and np.array_equal(a[..., 8:], q[..., 8:])
        assert np.allclose((a * b).sum(), (turn(q, 11) * turn(k, 0)).sum())


def test_plain_attention_against_torch():
    rng = np.random.default_rng(1)
    K, V = rng.standard_normal((5, 1, 16, 64)), rng.standard_normal((5, 1, 16, 64))
    q = rng.standard_normal((3, 2, 64))
    o, lse, _, _ = ref.prefix_attention(q, K, V, [4, 2], 20, np.array([[3, 0]]), [18], [0, 3], 0.2)
    flat = lambda A: torch.from_numpy(np.concatenate([A[4, 0], A[2, 0, :4], A[3, 0], A[0, 0, :2]]))
    s = torch.einsum("thd,jd->thj", torch.from_numpy(q), flat(K)) * 0.2
    s[0, :, 36:] = -torch.inf
    s[1, :, 37:] = -torch.inf
    assert np.allclose(o, (torch.softmax(s, -1) @ flat(V)).numpy()) and np.allclose(lse, torch.logsumexp(s, -1).numpy())


@pytest.mark.parametrize("code,change", [(NULL, dict(kv=None)), (NULL, dict(q=None)), (NULL, dict(n_free=None)), (NULL, dict(offs=None)), (NULL, dict(info=None)),
                                         (NULL, dict(pos=None)), (NULL, dict(slots=None)), (NULL, dict(free=None)), (UNSUPPORTED, dict(n_free=10 * P))])
def test_slots_refusals_without_requests(code, change):
    """a step of no requests writes its padding, offset and counts, so it needs where to"""
    assert rc(SLOTS, **dict(dict(B=0, kv_out=None, table=None), **change)) == code


@pytest.mark.parametrize("change", [dict(kv_out=2 * P), dict(kv_out=2 * P - 12), dict(offs=P), dict(offs=2 * P + 12), dict(offs=4 * P), dict(pos=P), dict(pos=8 * P, slots=8 * P + 28),
                                    dict(slots=2 * P - 4), dict(info=3 * P), dict(info=5 * P + 92), dict(table=P - 92), dict(table=3 * P + 32), dict(table=7 * P), dict(offs=9 * P),
                                    dict(kv_out=10 * P), dict(n_free=7 * P + 16), dict(n_free=8 * P), dict(n_free=6 * P), dict(n_free=5 * P + 4)])
def test_slots_refuses_arrays_that_share_memory(change):
    """what the call writes lies apart from all that it reads, and from all else that it writes"""
    assert rc(SLOTS, **change) == UNSUPPORTED
    assert b"overlaps" in osc.lib().osc_last_error()


def test_binding_refuses_tensors_in_host_memory():
    """a kernel given host addresses faults: calls whose tensors fit each other but lie on the CPU are refused"""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    h = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    slots = dict(kv_lens=i(3), q_lens=i(3), free_pages=i(9), n_free=i(1), block_table=i(3, 4), page_size=16, T=8)
    rope = dict(QKV=h(5, 768), Hq=4, Hkv=1, D=128, cos_sin=torch.zeros(9, 128), positions=i(5), slots=i(5), Kc=h(2, 1, 16, 128), Vc=h(2, 1, 16, 128))
    attn = dict(Q=h(5, 512), Hq=4, Hkv=1, D=128, Kc=h(4, 1, 16, 128), Vc=h(4, 1, 16, 128), prefix_pages=i(2), prefix_len=20, block_table=i(3, 4), kv_lens=i(3), q_offsets=i(4))
    for call in (lambda: osc.osc_page_slots(**slots), lambda: osc.osc_page_slots(**slots, out=(i(3), i(4), i(8), i(8), i(4))), lambda: osc.osc_qk_norm_rope(**rope),
                 lambda: osc.osc_qk_norm_rope(**rope, out=h(5, 512)), lambda: osc.osc_prefix_attention(**attn),
                 lambda: osc.osc_prefix_attention(**attn, workspace=torch.zeros(1 << 20, dtype=torch.uint8), out=(h(5, 512), None)),
                 lambda: osc.osc_rope_table(1e4, 64, 8, device="cpu"), lambda: osc.osc_rope_table(1e4, 64, 8, out=torch.zeros(8, 64))):
        with pytest.raises(AssertionError, match="GPU"):
            call()


def test_binding_refuses_other_types_of_16_bits():
    """fp16 is not read as if its bits were bf16; bits of bf16 in integers are (they go as far as the check that they are on the GPU)"""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    h = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    rope = dict(QKV=h(5, 768), Hq=4, Hkv=1, D=128, cos_sin=torch.zeros(9, 128), positions=i(5), slots=i(5), Kc=h(2, 1, 16, 128), Vc=h(2, 1, 16, 128), gamma_q=h(128),
                gamma_k=h(128), out=h(5, 512))
    attn = dict(Q=h(5, 512), Hq=4, Hkv=1, D=128, Kc=h(4, 1, 16, 128), Vc=h(4, 1, 16, 128), prefix_pages=i(2), prefix_len=20, block_table=i(3, 4), kv_lens=i(3), q_offsets=i(4))
    for call, good, names in ((osc.osc_qk_norm_rope, rope, ("QKV", "Kc", "Vc", "gamma_q", "gamma_k", "out")), (osc.osc_prefix_attention, attn, ("Q", "Kc", "Vc"))):
        for name in names:
            with pytest.raises(AssertionError, match="bf16"):
                call(**dict(good, **{name: good[name].half()}))
            for bits in (torch.uint16, torch.int16):
                with pytest.raises(AssertionError, match="GPU"):
                    call(**dict(good, **{name: good[name].view(bits)}))
    with pytest.raises(AssertionError, match="bf16"):
        osc.osc_prefix_attention(**attn, out=(h(5, 512).half(), None))


def test_binding_refuses_numbers_that_do_not_fit():
    """numbers past 32 bits are refused, not cut to some other number; a cache whose pages hold nothing is refused before anything is divided by its page size"""
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    h = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    wrap = 2 ** 32
    slots = dict(kv_lens=i(3), q_lens=i(3), free_pages=i(9), n_free=i(1), block_table=i(3, 4), page_size=16, T=8)
    for k, v in (("page_size", wrap + 16), ("page_size", -wrap + 16), ("pos_base", wrap), ("pos_base", 2 ** 31)):
        with pytest.raises(AssertionError, match="32 bits"):
            osc.osc_page_slots(**dict(slots, **{k: v}))
    rope = dict(QKV=h(5, 768), Hq=4, Hkv=1, D=128, cos_sin=torch.zeros(9, 128), positions=i(2, 5), slots=i(5), Kc=h(2, 1, 16, 128), Vc=h(2, 1, 16, 128), sections=[32, 32])
    for k, v in (("style", wrap + 1), ("sections", [wrap + 32, 32]), ("sections", [32, 32 - wrap])):
        with pytest.raises(AssertionError, match="32 bits"):
            osc.osc_qk_norm_rope(**dict(rope, **{k: v}))
    with pytest.raises(AssertionError, match="cos_sin"):
        osc.osc_qk_norm_rope(**dict(rope, cos_sin=torch.zeros(0, wrap + 128)))
    attn = dict(Q=h(5, 512), Hq=4, Hkv=1, D=128, Kc=h(4, 1, 16, 128), Vc=h(4, 1, 16, 128), prefix_pages=i(2), prefix_len=20, block_table=i(3, 4), kv_lens=i(3), q_offsets=i(4))
    for bad in (h(4, 1, 0, 128), h(0, 1, wrap + 16, 128)):
        with pytest.raises(AssertionError, match="cache"):
            osc.osc_prefix_attention(**dict(attn, Kc=bad, Vc=bad))
        with pytest.raises(AssertionError, match="cache"):
            osc.osc_qk_norm_rope(**dict(rope, Kc=bad, Vc=bad))
    for n in (2 ** 63 - 1, 2 ** 32):
        with pytest.raises(AssertionError, match="prefix_pages"):
            osc.osc_prefix_attention(**dict(attn, prefix_len=n))


@pytest.mark.parametrize("code,change", [(UNSUPPORTED, dict(P=2 ** 30 - 1)), (UNSUPPORTED, dict(P=2 ** 30 - 255)), (WORKSPACE, dict(P=2 ** 30 - 256))])
def test_attention_longest_prefix(code, change):
    """a prefix and 2^30 - 1 tokens of a request's own, with what the plan adds to them, are counted in 31 bits"""
    assert rc(ATTN, **change) == code


def test_workspace_size_as_documented():
    """the sizes that the header names, and none for a call that would be refused"""
    size = osc.osc_prefix_attention_workspace_bytes
    for mb, args in ((34, (1, 1, 32, 8, 128, 0)), (26, (1, 1, 24, 8, 64, 0)), (180, (64, 64, 32, 8, 128, 8192)), (103, (8192, 1, 32, 8, 128, 0)),
                     (227, (4000, 40, 32, 8, 128, 4096)), (770, (4000, 256, 32, 8, 128, 32700)), (1193, (8192, 8192, 32, 8, 128, 0))):
        assert round(size(*args) / 1e6) == mb, args
    for T, B, Hq, Hkv, D, P in ((2 ** 31, 4, 1, 1, 64, 0), (2 ** 27, 4, 32, 8, 128, 0), (2 ** 62, 1, 32, 8, 128, 0), (4, 8193, 8, 2, 128, 0), (4, 4, 8, 2, 128, 2 ** 30 - 255),
                                (4, 4, 8, 2, 128, 2 ** 62), (4, 4, 1024, 1024, 128, 0), (4, 4, 129, 1, 64, 0)):
        assert size(T, B, Hq, Hkv, D, P) == 0
        assert rc(ATTN, T=T, B=B, Hq=Hq, Hkv=Hkv, D=D, P=P, ldq=Hq * D, ldo=Hq * D) == UNSUPPORTED
