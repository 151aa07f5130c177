"""The attention layer of examples/attention_layer.py, step by step: prompts and single tokens behind a shared prompt, each step's
attention against double precision on the same cache, and against the same requests without a shared prefix.

Tolerances: as derived in test_gpu_attention.py, with the largest |v| in the place of the weighted average of |v|, which it bounds."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import attention_layer
    return attention_layer


@pytest.mark.parametrize("Hq,Hkv,D,ps", [(8, 2, 128, 16), (6, 3, 64, 32)])
def test_layer_steps(ex, Hq, Hkv, D, ps):
    layer = ex.Layer(hidden=512, Hq=Hq, Hkv=Hkv, D=D, pages=200, page_size=ps, max_pos=600)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rows = lambda n: torch.randn(n, layer.hidden, generator=g, device="cuda").bfloat16()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    shared = rows(45)
    free = torch.randperm(200, generator=g, device="cuda").to(torch.int32)
    prefix_pages, free = ex.prefill_prefix(layer, shared, free)
    batch = ex.Batch(layer, 4, 200, free, prefix_pages, 45)
    alone = ex.Layer(hidden=512, Hq=Hq, Hkv=Hkv, D=D, pages=200, page_size=ps, max_pos=600)  # the same weights, another cache
    apart = ex.Batch(alone, 4, 245, torch.arange(200, dtype=torch.int32, device="cuda"))
    apart.step(shared.repeat(4, 1), i32([45] * 4))
    for lens in ([7, 1, 0, 70], [1, 1, 1, 1], [1, 33, 5, 1], [1, 1, 1, 1]):
        x = rows(sum(lens))
        y, q, o, s = batch.step(x, i32(lens))
        assert s[4][2].item() == 0
        want = ex.plain_attention(layer, batch, q, s)
        top = layer.V.abs().max().double()
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * top
        assert ((o.double() - want).abs() <= tol).all()
        y2, q2, o2, s2 = apart.step(x, i32(lens))
        assert torch.equal(q, q2)  # positions follow the prefix, wherever it is kept
        assert ((o.double() - o2.double()).abs() <= 2 * tol).all()
        assert torch.isfinite(y).all() and y.shape == x.shape
    assert batch.kv_lens.tolist() == [10, 36, 7, 73] and apart.kv_lens.tolist() == [55, 81, 52, 118]


def test_pages_run_out(ex):
    """A request that finds no page is refused and told apart; the others go on, and what it kept stays valid."""
    layer = ex.Layer(hidden=512, Hq=4, Hkv=2, D=64, pages=8, page_size=16, max_pos=200)
    batch = ex.Batch(layer, 3, 64, torch.arange(4, dtype=torch.int32, device="cuda"))
    x = torch.randn(48, 512, device="cuda").bfloat16()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    _, _, _, s = batch.step(x, i32([16, 16, 16]))
    assert s[4].tolist() == [1, 3, 0, 48]
    _, q, o, s = batch.step(x[:3], i32([1, 1, 1]))  # each needs a new page, one is left
    assert s[4].tolist() == [0, 1, 2, 3] and s[0].tolist() == [17, 16, 16] and s[3].tolist()[1:] == [-1, -1]
    want = ex.plain_attention(layer, batch, q, s)
    assert ((o[0].double() - want[0]).abs() <= 2.0 ** -8 * want[0].abs() + 2.0 ** -7 * layer.V.abs().max()).all()


def test_shared_prompt_without_pages(ex):
    """A shared prompt that the cache cannot hold is an error, not a prefix of pages that nothing was written to."""
    layer = ex.Layer(hidden=512, Hq=4, Hkv=2, D=64, pages=8, page_size=16, max_pos=200)
    x = torch.randn(49, 512, device="cuda").bfloat16()
    free = torch.arange(5, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="4 pages, 3 are free"):
        ex.prefill_prefix(layer, x, free[:3])
    prefix_pages, left = ex.prefill_prefix(layer, x, free)
    assert sorted(prefix_pages.tolist() + left.tolist()) == [0, 1, 2, 3, 4] and prefix_pages.numel() == 4
