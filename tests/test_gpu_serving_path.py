"""The serving path of examples/paged_serving.py: prompt attention, compression,
pages and decoding together.

With the whole cache as the budget the compression keeps every entry, so each
step must equal causal attention over everything before it; with a smaller
budget a step must equal attention over the entries the cache really holds."""
import importlib.util
import math
import os

import pytest
import torch

from . import serving_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def ex():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    p = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_serving.py")
    spec = importlib.util.spec_from_file_location("paged_serving", p)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain(model, prompt, ys, base):
    """fp32 stack over [prompt; inputs of the steps] with fp64 attention: outputs of every row."""
    x = torch.cat([prompt, ys]).float()
    n = x.shape[0]
    pos = torch.arange(n)
    hidden = torch.arange(n)[None, :] > torch.arange(n)[:, None]
    for l in range(model.L):
        q, k, v = (t.cpu() for t in _project32(model, l, x))
        q, k = R.rotate(q, pos, base), R.rotate(k, pos, base)
        gq = model.Hq // model.G
        o = torch.stack([R.attend(q[:, h], k[:, h // gq], v[:, h // gq].double(), hidden)[0] for h in range(model.Hq)], 1)
        x = x + o.reshape(n, -1).float().to(x.device) @ model.o[l].float()
    return x


def _project32(model, l, x):
    n, G, Hq, d = x.shape[0], model.G, model.Hq, model.d
    q, k, v = (x @ model.qkv[l].float()).split([Hq * d, G * d, G * d], 1)
    return q.view(n, Hq, d), k.view(n, G, d), v.view(n, G, d)


@pytest.mark.parametrize("d", [64, 128])
def test_whole_budget_is_plain_attention(ex, d):
    # fp32: every difference is rounding.  A step's input is the step before's output, so the rows
    # are compared given the inputs the path itself used.
    model = ex.Stack(L=2, G=2, Hq=4, d=d, D=64, dtype=torch.float32, seed=1)
    g = torch.Generator(device="cuda").manual_seed(2)
    prompts = [torch.randn(n, 64, generator=g, device="cuda") for n in (150, 70)]
    steps, base = 3, 1.0e4
    x, y, cache, at = ex.serve(model, prompts, steps, ratio=1.0, rope_base=base, W=8, page_size=16)
    assert int(cache.lens.min()) == 70 + steps and int(cache.lens.max()) == 150 + steps
    assert at[:, 0].tolist() == [150, 151, 152]
    first = 0
    for b, p in enumerate(prompts):
        n = p.shape[0]
        inputs = torch.cat([x[first + n - 1:first + n], y[:-1, b]])
        want = plain(model, p, inputs, base)
        got = torch.cat([x[first:first + n], y[:, b]])
        # two layers of fp32 rounding on unit-sized streams
        assert float((got - want).abs().max()) < 2e-4
        first += n


def test_compressed_steps_attend_what_the_cache_holds(ex):
    model = ex.Stack(L=2, G=2, Hq=8, d=64, D=64, dtype=torch.bfloat16, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    prompts = [torch.randn(n, 64, generator=g, device="cuda").to(torch.bfloat16) for n in (600, 257)]
    steps = 5
    x, y, cache, at = ex.serve(model, prompts, steps, ratio=4.0, W=16, page_size=16)
    assert torch.isfinite(y.float()).all()
    lens = cache.lens.cpu()
    held = lens.sum() - steps * lens.numel()
    assert 0 < int(held) <= 4 * (600 + 257) // 4 and int(lens.min()) > steps
    # the last token's entries: log m = 0 and the rest as loaded; one more attention against fp64
    q = torch.randn(2, 8, 64, generator=g, device="cuda").to(torch.bfloat16)
    for l in range(2):
        out = cache.attention(l, q)
        want, tol = R.decode(q, cache.K, cache.V, cache.log_m, cache.table, cache.lens, l, bf16=True)
        assert ((out.double().cpu() - want).abs() <= tol).all()
        for b in range(2):
            for h in range(2):
                assert (R.entries(cache.log_m.cpu(), cache.table[l, b, h].cpu(), int(lens[l, b, h]))[-steps:] == 0).all()
    cache.status()
    assert math.isfinite(float(x.float().abs().max()))
