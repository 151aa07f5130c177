"""One attention layer of a serving loop on the library's kernels: RMSNorm with the quantiser, the q|k|v projection, cache pages
of the step's tokens, head norms with rotation and the write into the cache, attention behind a prompt that all requests share,
and the o projection.

    python examples/attention_layer.py [--requests 64] [--prefix 8192] [--steps 32]

Random weights of the 32-head, hidden 4096 configuration; prints microseconds a step, and how far one step's attention is from
the same rows computed plainly in double precision.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_12782_amd as osc  # noqa: E402

DEV = "cuda"


class Layer:
    """Weights, rotation angles and one paged cache.  Protected channels: one in every group of 32."""

    def __init__(self, hidden=4096, Hq=32, Hkv=8, D=128, pages=4096, page_size=64, max_pos=65536, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        rand = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=DEV) * std).bfloat16()
        self.hidden, self.Hq, self.Hkv, self.D, self.page_size = hidden, Hq, Hkv, D, page_size
        self.scale = D ** -0.5
        self.N = (Hq + 2 * Hkv) * D
        groups = torch.arange(hidden // 32, dtype=torch.int32, device=DEV)
        self.oidx_in = groups * 32 + torch.randint(0, 32, groups.shape, generator=g, device=DEV, dtype=torch.int32)
        groups = torch.arange(Hq * D // 32, dtype=torch.int32, device=DEV)
        self.oidx_out = groups * 32 + torch.randint(0, 32, groups.shape, generator=g, device=DEV, dtype=torch.int32)
        self.w_qkv = osc.osc_pack_weight(rand(self.N, hidden, std=hidden ** -0.5), self.oidx_in)
        self.w_o = osc.osc_pack_weight(rand(hidden, Hq * D, std=(Hq * D) ** -0.5), self.oidx_out)
        self.norm, self.norm_q, self.norm_k = 1 + rand(hidden, std=0.1), 1 + rand(D, std=0.1), 1 + rand(D, std=0.1)
        self.angles = osc.osc_rope_table(1e6, D, max_pos)
        self.K, self.V = (torch.zeros(pages, Hkv, page_size, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def forward(self, x, batch, slots_of_step):
        """x [T, hidden]: the step's rows, request by request -> (o projection's output, rows of queries, attention's output)"""
        kv_lens, q_offsets, positions, slots, _ = slots_of_step
        Xq, Xs, B, _ = osc.osc_rmsnorm_quantize_act(x, self.norm, 1e-6, self.oidx_in)
        qkv = osc.osc_dual_gemm(Xq, Xs, B, self.w_qkv, self.N, self.hidden, self.oidx_in.numel(), osc.OSC_DT_BF16)
        q = osc.osc_qk_norm_rope(qkv, self.Hq, self.Hkv, self.D, self.angles, positions, slots, self.K, self.V, self.norm_q, self.norm_k)
        o, _ = osc.osc_prefix_attention(q, self.Hq, self.Hkv, self.D, self.K, self.V, batch.prefix_pages, batch.prefix_len, batch.table, kv_lens, q_offsets,
                                        self.scale)
        Xq, Xs, B = osc.osc_quantize_act(o, self.oidx_out)
        y = osc.osc_dual_gemm(Xq, Xs, B, self.w_o, self.hidden, self.Hq * self.D, self.oidx_out.numel(), osc.OSC_DT_BF16)
        return y, q, o


class Batch:
    """Requests and the pages they hold; everything stays on the device."""

    def __init__(self, layer, requests, max_tokens, free_pages, prefix_pages=None, prefix_len=0):
        self.layer = layer
        self.kv_lens = torch.zeros(requests, dtype=torch.int32, device=DEV)
        self.table = torch.zeros(requests, -(-max_tokens // layer.page_size), dtype=torch.int32, device=DEV)
        self.free_pages, self.n_free = free_pages, torch.tensor([free_pages.numel()], dtype=torch.int32, device=DEV)
        self.prefix_pages = torch.zeros(0, dtype=torch.int32, device=DEV) if prefix_pages is None else prefix_pages
        self.prefix_len = prefix_len

    def step(self, x, q_lens):
        """x: rows of all requests, q_lens [requests] of them each"""
        s = osc.osc_page_slots(self.kv_lens, q_lens, self.free_pages, self.n_free, self.table, self.layer.page_size, x.shape[0], self.prefix_len)
        self.kv_lens, self.n_free = s[0], s[4][:1]
        return (*self.layer.forward(x, self, s), s)


def prefill_prefix(layer, x, free_pages):
    """The shared prompt, run as a single request: -> (its pages, the pages that are left)"""
    pages = -(-x.shape[0] // layer.page_size)
    if pages > free_pages.numel():
        raise ValueError(f"the shared prompt takes {pages} pages, {free_pages.numel()} are free")
    one = Batch(layer, 1, x.shape[0], free_pages)
    one.step(x, torch.tensor([x.shape[0]], dtype=torch.int32, device=DEV))
    return one.table[0, :pages].clone(), free_pages[:free_pages.numel() - pages]


def plain_attention(layer, batch, q, s):
    """the step's rows one by one in double precision"""
    G, D = layer.Hq // layer.Hkv, layer.D
    out = torch.zeros(q.shape[0], layer.Hq, D, dtype=torch.float64, device=DEV)
    lens, offs, ps = s[0].tolist(), s[1].tolist(), layer.page_size

    def rows(C, pages, n):
        j = torch.arange(n, device=DEV)
        return C[pages.long()[j // ps], :, j % ps].double()
    pk, pv = (rows(C, batch.prefix_pages, batch.prefix_len) for C in (layer.K, layer.V))
    for b, L in enumerate(lens):
        k, v = (torch.cat([p, rows(C, batch.table[b], L)]) for p, C in ((pk, layer.K), (pv, layer.V)))
        n = offs[b + 1] - offs[b]
        for i in range(n):
            m = batch.prefix_len + L - n + i + 1
            for h in range(layer.Hkv):
                qq = q[offs[b] + i].double().view(layer.Hq, D)[h * G:(h + 1) * G]
                out[offs[b] + i, h * G:(h + 1) * G] = torch.softmax(qq @ k[:m, h].t() * layer.scale, -1) @ v[:m, h]
    return out.view(q.shape[0], -1)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--requests", type=int, default=64)
    ap.add_argument("--prefix", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    layer = Layer(max_pos=a.prefix + a.steps + 64)
    free = torch.randperm(layer.K.shape[0], device=DEV).to(torch.int32)
    rows = lambda n: torch.randn(n, layer.hidden, device=DEV).bfloat16()
    prefix_pages, free = prefill_prefix(layer, rows(a.prefix), free)
    batch = Batch(layer, a.requests, a.steps + 16, free, prefix_pages, a.prefix)
    if a.requests * batch.table.shape[1] > free.numel():
        raise SystemExit(f"{a.requests} requests of {a.steps + 4} tokens take more than the {free.numel()} pages that are free")
    one = torch.ones(a.requests, dtype=torch.int32, device=DEV)
    x = rows(a.requests)
    for _ in range(4):
        y, q, o, s = batch.step(x, one)
    worst = (o.double() - plain_attention(layer, batch, q, s)).abs().max().item()
    start, end = torch.cuda.Event(True), torch.cuda.Event(True)
    start.record()
    for _ in range(a.steps):
        batch.step(x, one)
    end.record()
    torch.cuda.synchronize()
    print(f"{a.requests} requests behind {a.prefix} tokens: {start.elapsed_time(end) / a.steps * 1e3:.1f} us a step; "
          f"{batch.n_free.item()} pages free; attention against double precision: largest difference {worst:.2e} of {o.abs().max().item():.2f}")


if __name__ == "__main__":
    main()
