"""A run of the operators of speculative decoding together, as examples/speculative_decoding.py uses them: the tokens are those of decoding
one by one, the cache holds what it would hold then, pages come back; and a step in a graph, on a stream that is not the default one."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import speculative_decoding
    return speculative_decoding


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def cached(C, table, n):
    """keys (values) of a request's first n tokens, all layers"""
    ps = C.shape[3]
    j = torch.arange(n, device=DEV)
    return C[:, table.long()[j // ps], :, j % ps]


@pytest.mark.parametrize("Hq,Hkv,D,ps", [(8, 2, 128, 16), (6, 3, 64, 32)])
def test_same_tokens_as_one_by_one(ex, Hq, Hkv, D, ps):
    kw = dict(layers=2, hidden=512, Hq=Hq, Hkv=Hkv, D=D, vocab=1000, pages=200, page_size=ps, max_pos=600, seed=3)
    model, plain_model = ex.Model(**kw), ex.Model(**kw)
    B = 5
    prompts = torch.randint(0, 1000, (B, 13), device=DEV, dtype=torch.int32)
    batch, said, accepted = ex.decode(model, prompts, 10)
    counts = torch.stack(accepted)
    assert counts.min() >= 1 and counts.max() <= 5 and counts.float().mean() > 1.3  # some drafts are taken, some are not
    plain, one_by_one, _ = ex.decode(plain_model, prompts, int(max(len(s) for s in said)), [-1])
    for s, p in zip(said, one_by_one):
        assert s == p[:len(s)]
    lens = batch.kv_lens.tolist()
    assert lens == [12 + len(s) for s in said]  # the last token is known, not cached
    for C, P in ((model.K, plain_model.K), (model.V, plain_model.V)):
        for b, n in enumerate(lens):
            a, c = cached(C, batch.table[b], n), cached(P, plain.table[b], n)
            assert torch.equal(a[0], c[0])  # the first layer's depend on tokens and positions alone
            # bf16 results of sums in another order: a few roundings (2^-8) of the largest
            assert (a[1].float() - c[1].float()).abs().max() <= 2.0 ** -4 * c[1].float().abs().max()
    pages = sum(-(-n // ps) for n in lens)
    free = batch.free[:batch.n_free.item()].tolist()
    held = [p for b, n in enumerate(lens) for p in batch.table[b, :-(-n // ps)].tolist()]
    assert len(free) == 200 - pages and sorted(free + held) == list(range(200))


def test_pages_run_out(ex):
    """requests that find no pages accept nothing and keep their length; the others go on"""
    model = ex.Model(layers=1, hidden=512, Hq=4, Hkv=2, D=64, vocab=500, pages=8, page_size=16, max_pos=200)
    batch = ex.Batch(model, 3, 64, torch.arange(3, dtype=torch.int32, device=DEV))
    batch.prompts(torch.randint(0, 500, (3, 10), device=DEV, dtype=torch.int32))
    drafts, known = ex.Drafts(model, 3), batch.known
    path, accepted, _ = batch.step(drafts.rows(batch.known), drafts.parents, drafts.q_lens)  # each would need a second page
    assert accepted.tolist() == [0, 0, 0] and batch.kv_lens.tolist() == [10, 10, 10] and (path == -1).all() and batch.n_free.item() == 0
    assert torch.equal(batch.known, known)


def test_example_runs(ex, capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["speculative_decoding.py", "--requests", "4", "--steps", "3"])
    ex.main()
    assert "one by one: yes" in capsys.readouterr().out


def test_step_in_a_graph_and_on_a_stream(ex):
    """page slots, tree mask, attention, log probabilities, accepted path, moves, freed pages and forks: captured once and replayed on new lengths,
    trees and logits, each replay against the same calls made eagerly in between; outputs given, on a stream that is not the default one"""
    osc = ex.osc
    B, Hq, Hkv, D, ps, n, V, layers, P = 6, 8, 2, 128, 16, 9, 50001, 2, 20
    T, width, n_pages, N = B * n + 10, 12, 120, 3
    g = torch.Generator().manual_seed(1)
    Q = torch.randn(T, Hq * D, generator=g).bfloat16().to(DEV)
    prefix = i32([118, 119])
    kv, q = i32([0] * B), i32([n] * B)
    parents, tokens, logits = i32([0] * T), i32([0] * T), torch.zeros(T, V, device=DEV)
    src, dst = i32([0, 1, 0]), i32([3, 4, 5])
    ws = [torch.empty(osc.osc_tree_attention_workspace_bytes(T, B, Hq, Hkv, D, P), dtype=torch.uint8, device=DEV),
          torch.empty(osc.osc_token_logprobs_workspace_bytes(T, V, 5), dtype=torch.uint8, device=DEV)]

    def state(seed):
        gen = torch.Generator().manual_seed(seed)
        return dict(table=i32(np.arange(B * width).reshape(B, width)), free=i32(np.arange(72, 118)), n_free=i32([40]), refs=i32(np.zeros(n_pages)),
                    K=torch.randn(layers, n_pages, Hkv, ps, D, generator=gen).bfloat16().to(DEV), V=torch.randn(layers, n_pages, Hkv, ps, D, generator=gen).bfloat16().to(DEV))

    def step(s):
        lens, offs, _, slots, info = osc.osc_page_slots(kv, q, s["free"], s["n_free"], s["table"], ps, T)
        mask, pos = osc.osc_tree_mask(parents, offs, lens, 1, P)
        o, lse = osc.osc_tree_attention(Q, Hq, Hkv, D, s["K"][0], s["V"][0], prefix, P, s["table"], lens, offs, mask, want_lse=True, workspace=ws[0])
        res = osc.osc_token_logprobs(logits, tokens, 5, workspace=ws[1])
        acc = osc.osc_tree_accept(parents, tokens, res[1][:, 0], offs, lens, slots)
        osc.osc_cache_move(s["K"], s["V"], acc[4], slots, offs)
        freed = osc.osc_page_free(lens, acc[3], s["table"], s["free"], info[:1], ps, s["refs"])
        after = acc[3] + 0
        a, b, forked = osc.osc_page_fork(src, dst, after, s["table"], s["refs"], s["free"], freed[:1], ps)
        osc.osc_cache_move(s["K"], s["V"], a, b)
        return lens, offs, slots, info, mask, pos, o, lse, *res, *acc, freed, after, a, b, forked
    stream = torch.cuda.Stream()
    live = state(0)
    with torch.cuda.stream(stream):
        step(live)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs = step(live)
        gen = np.random.default_rng(0)
        for k in range(5):
            kv.copy_(i32(np.concatenate([gen.integers(0, 60, 3), gen.integers(0, 9, 3)])))
            q.copy_(i32(gen.integers(1, n + 1, B)))
            parents.copy_(i32(np.where(gen.random(T) < 0.6, np.arange(T) % n - 1, 0)))
            tokens.copy_(i32(gen.integers(0, 4, T)))
            logits.copy_(torch.randn(T, V, generator=g))
            logits[:, :4] += 9 * torch.rand(T, 4, generator=g).to(DEV)
            Q.copy_(torch.randn(Q.shape, generator=g).bfloat16())
            fresh = state(k + 1)
            for name in live:
                live[name].copy_(fresh[name])
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in outs]
            eager = step(fresh)
            stream.synchronize()
            rows = int(eager[1][-1])
            assert eager[17].max() > 1 and eager[-1][2] == 0
            for i, (a, b) in enumerate(zip(got, eager)):
                a, b = (a[:rows], b[:rows]) if i in (6, 7) else (a, b)  # rows of no request are left as they are
                assert torch.equal(a, b), (k, i)
            for name in live:
                assert torch.equal(live[name], fresh[name]), name


def test_nothing_is_allocated_where_outputs_are_given(ex):
    osc = ex.osc
    T, B = 12, 2
    parents, offs, kv, slots = i32([-1, 0, 0, 1, 1, 2] * 2), i32([0, 6, 12]), i32([9, 30]), i32(np.arange(12))
    tok, table, free, refs = i32(np.zeros(12)), i32([[0, 1], [2, 3]]), i32(np.arange(4, 40)), i32(np.zeros(40))
    K, V = (torch.zeros(40, 1, 16, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    x = torch.randn(T, 70000, device=DEV)
    new = lambda: (osc.osc_tree_mask(parents, offs, kv), osc.osc_tree_accept(parents, tok, tok, offs, kv, slots), osc.osc_token_logprobs(x, tok, 3),
                   osc.osc_page_fork(i32([0]), i32([1]), kv.clone(), table.clone(), refs.clone(), free, i32([9]), 16))
    m, acc, lp, fk = new()
    info, one, two, n_free, lens = torch.empty(4, dtype=torch.int32, device=DEV), i32([0]), i32([1]), i32([9]), kv.clone()
    ws = torch.empty(osc.osc_token_logprobs_workspace_bytes(T, 70000, 3), dtype=torch.uint8, device=DEV)
    wa = torch.empty(osc.osc_tree_attention_workspace_bytes(T, B, 2, 1, 64, 0), dtype=torch.uint8, device=DEV)
    Q, o, lse, none = torch.randn(T, 128, device=DEV).bfloat16(), torch.empty(T, 128, dtype=torch.bfloat16, device=DEV), torch.empty(T, 2, device=DEV), i32([])
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    osc.osc_tree_mask(parents, offs, kv, out=m)
    osc.osc_tree_attention(Q, 2, 1, 64, K, V, none, 0, table, kv, offs, m[0], workspace=wa, out=(o, lse))
    osc.osc_tree_accept(parents, tok, tok, offs, kv, slots, out=acc)
    osc.osc_cache_move(K, V, acc[4], slots, offs)
    osc.osc_page_free(kv, acc[3], table, free, n_free, 16, refs, out=info)
    osc.osc_page_fork(one, two, lens, table, refs, free, n_free, 16, out=fk)
    osc.osc_token_logprobs(x, tok, 3, workspace=ws, out=lp)
    torch.cuda.synchronize()
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
