"""The path of examples/shared_context.py: contexts compressed into quantised pages,
questions that share them, requests that leave and come back, together.

With the whole context kept in pages of the rows' type each step must equal causal
attention over the context and everything of its own before it; otherwise attention
over the entries that the caches really hold."""
import importlib.util
import os

import pytest
import torch

from . import quant_reference as Q
from . import serving_reference as R
from .test_gpu_serving_path import plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def ex():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    p = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_context.py")
    spec = importlib.util.spec_from_file_location("shared_context", p)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def inputs(ex, dtype, d, seed, contexts, questions, D=64):
    model = ex.Stack(L=2, G=2, Hq=4, d=d, D=D, dtype=dtype, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)

    def some(n):
        return torch.randn(n, D, generator=g, device="cuda").to(dtype)
    return model, [some(n) for n in contexts], [[some(n) for n in qs] for qs in questions]


@pytest.mark.parametrize("d", [64, 128])
def test_whole_contexts_are_plain_attention(ex, d):
    # fp32 pages and every entry kept: all differences are rounding, given the inputs that the steps used
    model, contexts, questions = inputs(ex, F32, d, 1, (150, 70), [(3, 1, 5), (2,)])
    ins, outs, cache, prefix, at = ex.serve(model, contexts, questions, 7, ratio=1.0, W=8, page_size=16, quantised=False, pause=4)
    assert prefix.lens[0, :, 0].tolist() == [150, 70] and (cache.lens == 7).all()
    assert at[:, 0].tolist() == list(range(150, 157)) and at[0].tolist() == [150, 150, 150, 70]
    b = 0
    for x, qs in zip(contexts, questions):
        for q in qs:
            assert torch.equal(ins[:q.shape[0], b], q) and torch.equal(ins[q.shape[0]:, b], outs[q.shape[0] - 1:-1, b])
            want = plain(model, x, ins[:, b], 1.0e4)[x.shape[0]:]
            # two layers of fp32 rounding on unit-sized streams
            assert float((outs[:, b] - want).abs().max()) < 2e-4
            b += 1


@pytest.mark.parametrize("dtype,quantised", [(BF, True), (F32, True), (BF, False)])
def test_requests_that_leave_and_come_back(ex, dtype, quantised):
    # nothing is lost on the way, and the order of the sums is that of the entries: the same bits
    model, contexts, questions = inputs(ex, dtype, 64, 5, (300, 90), [(3, 2), (1, 4, 2)])
    run = [ex.serve(model, contexts, questions, 21, ratio=3.0, page_size=16, quantised=quantised, pause=p) for p in (None, 18)]
    (_, a, c0, _, _), (_, b, c1, _, _) = run
    assert torch.isfinite(a.float()).all() and torch.equal(a, b) and torch.equal(c0.lens, c1.lens)
    assert not torch.equal(c0.table, c1.table)
    for r in range(5):
        one, two = c0.unload(r), c1.unload(r)
        assert all(torch.equal(getattr(one, f), getattr(two, f)) for f in ("K", "V", "log_m", "offsets"))


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64)])
def test_compressed_steps_attend_what_the_caches_hold(ex, dtype, d):
    model, contexts, questions = inputs(ex, dtype, d, 9, (700, 330), [(4, 3, 2), (2, 6)])
    ins, outs, cache, prefix, _ = ex.serve(model, contexts, questions, 6, ratio=4.0, page_size=16)
    assert cache.quantised and prefix.quantised and torch.isfinite(outs.float()).all()
    assert 0 < int(prefix.lens.sum()) <= 4 * (700 + 330) // 4
    q = torch.randn(5, 4, d, device="cuda").to(dtype)
    cu = torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda")
    attend = ex.gk.SharedAttention(cache, prefix)
    bits = R.BITS_BF16 if dtype is BF else R.BITS_F32
    pools = [[torch.from_numpy(Q.values(x, s)) for x, s in ((c.K, c.k_scale), (c.V, c.v_scale))] + [c.log_m.cpu().double()]
             for c in (prefix, cache)]
    for l in range(2):
        out = attend(l, q, cu).double().cpu()
        for b in range(5):
            for g in range(2):
                rows = [[R.entries(x, c.table[l, i, g].cpu(), int(c.lens[l, i, g])) for x in pool]
                        for pool, c, i in ((pools[0], prefix, int(b >= 3)), (pools[1], cache, b))]
                k, v, m = (torch.cat(x) for x in zip(*rows))
                at = slice(2 * g, 2 * g + 2)
                o, _, w = R.attend(q[b, at].double().cpu(), k, v, bias=m)
                # weights of the prefix's entries are rounded to f16 (11 bits), values below 2^-33 of the largest are 0
                tol = R.attend_bound(q[b, at].double().cpu(), k, v, o, w, weight_bits=11 if dtype is BF else R.BITS_F32, out_bits=bits)
                tol = tol + (2.0 ** -22 * float(m.abs().max()) + 2.0 ** -32) * float(v.abs().max())
                assert ((out[b, at] - o).abs() <= tol).all()
    attend.status()
