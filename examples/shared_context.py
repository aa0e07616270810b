"""Many questions on a few long contexts, on one GPU.

    python examples/shared_context.py

The attention stack of ``paged_serving.py`` again.  Every context is kept once and
serves all its questions:

1. a context's tokens are stored and attended (``PagedCache.append``,
   ``PromptAttention``), compressed (``Compressor``) and loaded into a slot of a
   prefix cache, with ``quantised=True`` as e4m3 codes and a scale a row;
2. the questions of context p are requests ``cu_prefix[p]`` to ``cu_prefix[p + 1]``
   of a cache of their own, without entries at first.  Every step takes a token of
   each, of its question as long as there are any and its last output after that:
   ``advance``, then per layer ``append`` and ``SharedAttention``;
3. at step ``pause`` the requests leave the GPU's pages (``unload``, ``release``) and
   come back into other ones (``load``), as after a wait for memory.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paged_serving import Stack  # noqa: E402
from paper_2608_07001_gb300 import gracekv as gk  # noqa: E402


def prefill(model, x, rope_base):
    """x [T, D] through the stack: (K, V [L, G, T, d], the layers' queries [Hq, T, d])."""
    L, G, Hq, d, dt, dev, T = model.L, model.G, model.Hq, model.d, model.dtype, x.device, x.shape[0]
    i32 = dict(dtype=torch.int32, device=dev)
    K, V = (torch.empty(L, G, T, d, dtype=dt, device=dev) for _ in range(2))
    dense = gk.PagedCache(K.view(L * G, T, d), V.view(L * G, T, d), torch.arange(L * G, **i32).view(L, 1, G, 1),
                          torch.full((L, 1, G), T, **i32), Hq=Hq, rope_base=rope_base)
    attend = gk.PromptAttention(G=G, Hq=Hq, d=d, dtype=dt, device=dev)
    pos, whole, seen = torch.arange(T, **i32), torch.tensor([0, T], **i32), []
    for l in range(L):
        q, k, v = model.project(l, x)
        q = dense.append(l, k, v, pos, q=q, cu_new=whole)
        x = model.mix(l, x, attend(q, K[l].transpose(0, 1), V[l].transpose(0, 1), whole))
        seen.append(q.transpose(0, 1))
    attend.status()
    dense.status()
    return K, V, seen


def serve(model, contexts, questions, steps, *, ratio=4.0, rope_base=1.0e4, W=16, page_size=32, quantised=True, pause=None):
    """contexts: a list of [T_p, D] embeddings; questions: for each one a list of [n, D].
    Returns (inputs and outputs of every step [steps, B, D], the requests' cache, the
    prefix cache, the positions of the steps [steps, B])."""
    L, G, Hq, d, dt, dev = model.L, model.G, model.Hq, model.d, model.dtype, contexts[0].device
    P, flat = len(contexts), [q for qs in questions for q in qs]
    B = len(flat)
    T = [c.shape[0] for c in contexts]
    base = [T[p] for p, qs in enumerate(questions) for _ in qs]
    starts = [0]
    for qs in questions:
        starts.append(starts[-1] + len(qs))
    cu_prefix = torch.tensor(starts, dtype=torch.int32, device=dev)

    # 1. the contexts
    own = dict(L=L, G=G, Hq=Hq, d=d, dtype=dt, page_size=page_size, device=dev, quantised=quantised)
    budgets = [gk.gracekv_budget_for_ratio(L, G, n, ratio) for n in T]
    prefix = gk.PagedCache.allocate(B=P, max_pages=-(-max(T) // page_size),
                                    n_pages=sum(b // page_size + L * G for b in budgets), **own)
    for p, x in enumerate(contexts):
        K, V, seen = prefill(model, x, rope_base)
        w = min(W, T[p])
        comp = gk.Compressor(gk.make_params(L, G, Hq, T[p], d, w, dtype=dt, budget=budgets[p], rope_base=rope_base), device=dev)
        packed = comp(K, V, torch.stack([q[:, T[p] - w:] for q in seen]).contiguous())
        prefix.load(p, packed, comp.n_entries)
    prefix.status()

    # 2. the questions; their keys are rotated to positions behind the whole context
    per = -(-steps // page_size)
    cache = gk.PagedCache.allocate(B=B, max_pages=per, n_pages=L * B * G * per, rope_base=rope_base, **own)
    attend = gk.SharedAttention(cache, prefix)
    asked = torch.tensor([q.shape[0] for q in flat], device=dev)[:, None]
    tokens = torch.zeros(steps, B, model.D, dtype=dt, device=dev)
    for b, q in enumerate(flat):
        n = min(steps, q.shape[0])
        tokens[:n, b] = q[:n]
    ins, outs, at, y = [], [], [], tokens[0]
    for s in range(steps):
        if s == pause:
            away = [cache.unload(b) for b in range(B)]
            for b in range(B):
                cache.release(b)
            for b in reversed(range(B)):                   # in another order: other pages
                cache.load(b, away[b], away[b].K.shape[0])
        cache.advance([1] * B if s == 0 else None)
        pos = torch.tensor([n + s for n in base], dtype=torch.int32, device=dev)
        x = torch.where(asked > s, tokens[s], y)
        ins.append(x)
        for l in range(L):
            q, k, v = model.project(l, x)
            q = cache.append(l, k, v, pos, q=q)
            x = model.mix(l, x, attend(l, q, cu_prefix))
        y = x
        outs.append(y)
        at.append(pos)
    attend.status()
    cache.status()
    return torch.stack(ins), torch.stack(outs), cache, prefix, torch.stack(at)


def main():
    torch.manual_seed(0)
    model = Stack()

    def some(n):
        return torch.randn(n, model.D, device="cuda").to(model.dtype)

    contexts = [some(n) for n in (3000, 1700)]
    questions = [[some(n) for n in (12, 7, 30, 9)], [some(n) for n in (5, 21)]]
    _, y, cache, prefix, _ = serve(model, contexts, questions, steps=40, pause=20)
    full, kept = sum(c.shape[0] for c in contexts) * model.L * model.G, int(prefix.lens.sum())
    held = sum(t.numel() * t.element_size() for t in prefix._pool[:2]) + sum(t.numel() for t in prefix._pool[-2:])
    print(f"{len(contexts)} contexts, {kept} of {full} entries kept in {held} bytes of codes and scales; "
          f"{y.shape[1]} requests, {y.shape[0]} steps, {cache.n_pages - cache._n_free} of {cache.n_pages} pages used")


if __name__ == "__main__":
    main()
