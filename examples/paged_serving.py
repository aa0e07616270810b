"""Several requests from their prompts to decoded tokens, on one GPU.

    python examples/paged_serving.py

A small attention stack with random weights stands in for a model: per layer a
fused q/k/v projection, attention, an output projection added to the stream.
The path is the one a server takes:

1. the prompts of all requests, packed: per layer the keys and queries are
   rotated and the keys and values stored ([L, G, N, d], one page a KV head) by
   ``PagedCache.append``, and attended by ``PromptAttention``;
2. each request's cache is compressed (``Compressor``), its last ``W`` queries
   as the observation window;
3. the packed caches become pages of one shared pool (``PagedCache.load``);
4. every step adds one token per request: ``advance`` once, then per layer
   ``append`` (rotation on the way into the pages) and ``attention``.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_07001_gb300 import gracekv as gk  # noqa: E402


class Stack:
    """Random weights of L attention layers."""

    def __init__(self, L=2, G=2, Hq=8, d=128, D=256, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.L, self.G, self.Hq, self.d, self.D, self.dtype = L, G, Hq, d, D, dtype

        def weight(n, m):
            return (torch.randn(n, m, generator=g, device=device) / n ** 0.5).to(dtype)

        self.qkv = [weight(D, (Hq + 2 * G) * d) for _ in range(L)]
        self.o = [weight(Hq * d, D) for _ in range(L)]

    def project(self, l, x):
        """x [N, D] -> q [N, Hq, d], k and v [N, G, d], slices of one projection."""
        n, G, Hq, d = x.shape[0], self.G, self.Hq, self.d
        q, k, v = (x @ self.qkv[l]).split([Hq * d, G * d, G * d], dim=1)
        return q.view(n, Hq, d), k.view(n, G, d), v.view(n, G, d)

    def mix(self, l, x, attended):
        return x + attended.reshape(x.shape[0], -1).to(self.dtype) @ self.o[l]


def serve(model, prompts, steps, ratio=4.0, rope_base=1.0e4, W=16, page_size=32):
    """prompts: a list of [T_b, D] embeddings.  Returns (prompt outputs [N, D],
    decoded outputs [steps, B, D], the paged cache, positions of the steps [steps, B])."""
    L, G, Hq, d, dt, dev = model.L, model.G, model.Hq, model.d, model.dtype, prompts[0].device
    T = [p.shape[0] for p in prompts]
    B, N = len(T), sum(T)
    bounds = [0]
    for n in T:
        bounds.append(bounds[-1] + n)
    i32 = dict(dtype=torch.int32, device=dev)
    cu = torch.tensor(bounds, **i32)

    # 1. the prompts, packed; a dense cache is a paged one with a page a KV head
    K, V = (torch.empty(L, G, N, d, dtype=dt, device=dev) for _ in range(2))
    dense = gk.PagedCache(K.view(L * G, N, d), V.view(L * G, N, d), torch.arange(L * G, **i32).view(L, 1, G, 1),
                          torch.full((L, 1, G), N, **i32), Hq=Hq, rope_base=rope_base)
    attend = gk.PromptAttention(G=G, Hq=Hq, d=d, dtype=dt, device=dev)
    pos = torch.cat([torch.arange(n, **i32) for n in T])
    whole = torch.tensor([0, N], **i32)
    x = torch.cat(prompts)
    seen = []
    for l in range(L):
        q, k, v = model.project(l, x)
        q = dense.append(l, k, v, pos, q=q, cu_new=whole)
        x = model.mix(l, x, attend(q, K[l].transpose(0, 1), V[l].transpose(0, 1), cu))
        seen.append(q)
    attend.status()
    dense.status()

    # 2. and 3. every request compressed and moved into the shared pages
    budgets = [gk.gracekv_budget_for_ratio(L, G, n, ratio) for n in T]
    most = max(T) + steps
    cache = gk.PagedCache.allocate(L=L, B=B, G=G, Hq=Hq, d=d, dtype=dt, page_size=page_size, rope_base=rope_base,
                                   max_pages=-(-most // page_size),
                                   n_pages=sum(b // page_size + L * G * (2 + steps // page_size) for b in budgets), device=dev)
    for b, n in enumerate(T):
        a, e = bounds[b], bounds[b + 1]
        w = min(W, n)
        Q = torch.stack([q[e - w:e].transpose(0, 1) for q in seen]).contiguous()         # [L, Hq, W, d]
        comp = gk.Compressor(gk.make_params(L, G, Hq, n, d, w, dtype=dt, budget=budgets[b], rope_base=rope_base), device=dev)
        packed = comp(K[:, :, a:e].contiguous(), V[:, :, a:e].contiguous(), Q)
        cache.load(b, packed, comp.n_entries)

    # 4. one token per request and step; the last prompt output is the first input
    y = x[torch.tensor(bounds[1:], device=dev) - 1]
    outs, at = [], []
    for s in range(steps):
        pos = torch.tensor([n + s for n in T], **i32)
        cache.advance()
        for l in range(L):
            q, k, v = model.project(l, y)
            q = cache.append(l, k, v, pos, q=q)
            y = model.mix(l, y, cache.attention(l, q))
        outs.append(y)
        at.append(pos)
    cache.status()
    return x, torch.stack(outs), cache, torch.stack(at)


def main():
    torch.manual_seed(0)
    model = Stack()
    prompts = [torch.randn(n, model.D, device="cuda").to(model.dtype) for n in (700, 1500, 433)]
    x, y, cache, _ = serve(model, prompts, steps=20)
    full, kept = sum(p.shape[0] for p in prompts) * model.L * model.G, int(cache.lens.sum()) - 20 * len(prompts) * model.L * model.G
    print(f"{len(prompts)} prompts, {x.shape[0]} tokens; {kept} of {full} cache entries kept; {y.shape[0]} steps, "
          f"entries per (layer, request, head) {int(cache.lens.min())}..{int(cache.lens.max())}, "
          f"{cache.n_pages - cache._n_free} of {cache.n_pages} pages used")


if __name__ == "__main__":
    main()
