"""Speculative decoding on the library's kernels: every step scores a tree of drafted tokens of each request, keeps the path that the model
agrees with and gives the other tokens' cache back; no length, token or page number is read by the host.

    python examples/speculative_decoding.py [--requests 32] [--steps 24] [--no-drafts]

A small model of random weights whose head is made so that a token mostly has one successor, and drafts that guess it three times in
four.  Prints accepted tokens and microseconds a step, the entropy of the choices, and whether the tokens are those of decoding one by one.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2604_12782_amd as osc  # noqa: E402
from attention_layer import DEV, Layer  # noqa: E402

i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)

# a known token, then at every depth the draft and an alternative beside it
TREE = [-1, 0, 0, 1, 1, 3, 3, 5, 5]


class Model:
    """Attention layers with one cache [layers, pages, Hkv, page_size, D], token embeddings and a head."""

    def __init__(self, layers=2, hidden=1024, Hq=8, Hkv=2, D=128, vocab=4096, pages=1024, page_size=16, max_pos=4096, seed=0):
        self.layers = [Layer(hidden, Hq, Hkv, D, 1, page_size, max_pos, seed + i) for i in range(layers)]
        self.K, self.V = (torch.zeros(layers, pages, Hkv, page_size, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        g = torch.Generator(device=DEV)
        g.manual_seed(seed + 100)
        self.embedding = torch.randn(vocab, hidden, generator=g, device=DEV).bfloat16()
        self.successor = torch.randperm(vocab, generator=g, device=DEV)
        head = torch.empty_like(self.embedding)
        head[self.successor] = self.embedding * (0.4 * hidden ** -0.5)
        self.norm = torch.ones(hidden, dtype=torch.bfloat16, device=DEV)
        self.oidx = self.layers[0].oidx_in
        self.head = osc.osc_pack_weight(head, self.oidx)
        self.vocab, self.hidden, self.page_size = vocab, hidden, page_size

    def logits(self, tokens, positions, slots, attention):
        """rows of tokens -> float32 [T, vocab]; attention(layer, queries, K, V) of one layer"""
        x = self.embedding[tokens.long()]
        for i, m in enumerate(self.layers):
            Xq, Xs, B, _ = osc.osc_rmsnorm_quantize_act(x, m.norm, 1e-6, m.oidx_in)
            qkv = osc.osc_dual_gemm(Xq, Xs, B, m.w_qkv, m.N, m.hidden, m.oidx_in.numel(), osc.OSC_DT_BF16)
            q = osc.osc_qk_norm_rope(qkv, m.Hq, m.Hkv, m.D, m.angles, positions, slots, self.K[i], self.V[i], m.norm_q, m.norm_k)
            Xq, Xs, B = osc.osc_quantize_act(attention(m, q, self.K[i], self.V[i]), m.oidx_out)
            x = x + 0.25 * osc.osc_dual_gemm(Xq, Xs, B, m.w_o, m.hidden, m.Hq * m.D, m.oidx_out.numel(), osc.OSC_DT_BF16)
        Xq, Xs, B, _ = osc.osc_rmsnorm_quantize_act(x, self.norm, 1e-6, self.oidx)
        return osc.osc_dual_gemm(Xq, Xs, B, self.head, self.vocab, self.hidden, self.oidx.numel(), osc.OSC_DT_F32)


class Batch:
    """Requests, their pages, and the token of each that is known but not cached yet."""

    def __init__(self, model, requests, max_tokens, pages=None):
        self.model = model
        self.kv_lens = i32([0] * requests)
        self.table = torch.zeros(requests, -(-max_tokens // model.page_size), dtype=torch.int32, device=DEV)
        self.free = torch.randperm(model.K.shape[1], device=DEV).to(torch.int32) if pages is None else pages
        self.n_free = i32([self.free.numel()])
        self.known = None

    def step(self, tokens, parents, q_lens, given=None):
        """Rows `tokens`, request by request: each request's known token, then its drafts, continuing rows `parents`.  `given`: rows' tokens where a
        prompt's are -1 (accepted as they are) -> (path, accepted, logits' results)"""
        m, ps = self.model, self.model.page_size
        lens, offsets, _, slots, info = osc.osc_page_slots(self.kv_lens, q_lens, self.free, self.n_free, self.table, ps, tokens.numel())
        mask, positions = osc.osc_tree_mask(parents, offsets, lens)
        attention = lambda a, q, K, V: osc.osc_tree_attention(q, a.Hq, a.Hkv, a.D, K, V, i32([]), 0, self.table, lens, offsets, mask, a.scale)[0]
        results = osc.osc_token_logprobs(m.logits(tokens, positions, slots, attention), None, 1)
        path, accepted, known, self.kv_lens, src = osc.osc_tree_accept(parents, tokens if given is None else given, results[1][:, 0], offsets, lens, slots)
        self.known = known if self.known is None else torch.where(accepted > 0, known, self.known)  # a request without pages goes on where it was
        osc.osc_cache_move(m.K, m.V, src, slots, offsets)
        self.n_free = osc.osc_page_free(lens, self.kv_lens, self.table, self.free, info[:1], ps, None, m.K.shape[1])[:1]
        return path, accepted, results

    def prompts(self, tokens):
        """[requests, n]: all of them are accepted, whatever the model would have chosen"""
        B, n = tokens.shape
        chain = torch.arange(-1, n - 1, dtype=torch.int32, device=DEV).repeat(B)
        return self.step(tokens.reshape(-1), chain, i32([n] * B), torch.full((B * n,), -1, dtype=torch.int32, device=DEV))


class Drafts:
    """Trees of guesses: right three times in four, the alternatives every second time."""

    def __init__(self, model, requests, tree=TREE, seed=1):
        self.model, self.tree, self.requests = model, tree, requests
        self.parents = i32(tree).repeat(requests)
        self.q_lens = i32([len(tree)] * requests)
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)

    def rows(self, known):
        """-> int32 [requests * len(tree)]"""
        out = torch.empty(self.requests, len(self.tree), dtype=torch.int32, device=DEV)
        out[:, 0] = known
        for i, p in enumerate(self.tree[1:], 1):
            right = torch.rand(self.requests, generator=self.gen, device=DEV) < (0.75 if i == p + 1 or i % 2 else 0.5)
            wrong = torch.randint(0, self.model.vocab, (self.requests,), generator=self.gen, device=DEV)
            out[:, i] = torch.where(right, self.model.successor[out[:, p].long()], wrong).int()
        return out.view(-1)


def decode(model, prompts, steps, tree=TREE, seed=1, pages=None):
    """-> (batch, the tokens of every request after its prompt, a list each; accepted tokens of every step)"""
    B = prompts.shape[0]
    batch = Batch(model, B, prompts.shape[1] + (steps + 2) * len(tree), pages)
    batch.prompts(prompts)
    drafts = Drafts(model, B, tree, seed)
    first, log = batch.known, []
    for _ in range(steps):
        rows = drafts.rows(batch.known)
        path, accepted, _ = batch.step(rows, drafts.parents, drafts.q_lens)
        log.append((rows, path, accepted, batch.known))
    said = [[t] for t in first.tolist()]
    for rows, path, accepted, known in log:  # read back once, after the last step
        rows, path, accepted, known = (t.tolist() for t in (rows, path, accepted, known))
        for b in range(B):
            at = b * len(tree)
            if accepted[b]:
                said[b] += [rows[at + i] for i in path[at + 1:at + accepted[b]]] + [known[b]]
    return batch, said, [x[2] for x in log]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=32)
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--no-drafts", action="store_true", help="decode one by one")
    a = ap.parse_args()
    tree = [-1] if a.no_drafts else TREE
    model = Model()
    need = a.requests * -(-(20 + (a.steps + 2) * max(len(tree), len(TREE))) // model.page_size)
    if need > model.K.shape[1]:
        raise SystemExit(f"{a.requests} requests of {a.steps} steps may take {need} pages, the cache has {model.K.shape[1]}")
    prompts = torch.randint(0, model.vocab, (a.requests, 20), device=DEV, dtype=torch.int32)
    _, said, accepted = decode(model, prompts, a.steps, tree)
    _, plain, _ = decode(model, prompts, a.steps, [-1])
    batch = Batch(model, a.requests, 20 + (a.steps + 2) * len(tree))
    batch.prompts(prompts)
    drafts = Drafts(model, a.requests, tree)
    start, end = torch.cuda.Event(True), torch.cuda.Event(True)
    rows = drafts.rows(batch.known)
    start.record()
    for _ in range(a.steps):
        _, _, results = batch.step(rows, drafts.parents, drafts.q_lens)
    end.record()
    torch.cuda.synchronize()
    rate = torch.stack(accepted).float().mean().item()
    same = all(s[:len(p)] == p[:len(s)] for s, p in zip(said, plain))
    print(f"{a.requests} requests, trees of {len(tree)} tokens: {rate:.2f} tokens a step, {start.elapsed_time(end) / a.steps * 1e3:.0f} us a step; "
          f"entropy of the choices {results[4].mean().item():.2f}; the tokens of decoding one by one: {'yes' if same else 'NO'}")


if __name__ == "__main__":
    main()
