"""Logits of billions: the weight is on one key and nothing overflows on the way
to it, or the row is NaN; never a wrong finite row."""
import math

import numpy as np
import pytest
import torch

from . import serving_reference as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


def one_channel(n, keys, d, dtype, sign, scale):
    """q, k of one channel of powers of two: the products are exact, and all scores differ by 2^-8 of themselves or
    more, so that every query's weight is on one key (on equal keys, where sizes repeat).  x [keys]: the logits."""
    per = 128
    size = torch.tensor([2.0 ** (i // per) * (1 + (i % per) / per) for i in range(min(keys, 1024))])
    order = torch.randperm(len(size), generator=torch.Generator().manual_seed(n))
    at = order.repeat(-(-keys // len(size)))[:keys]
    q, k = torch.zeros(n, 4, d), torch.zeros(keys, 2, d)
    q[:, :, 5] = 2.0 ** 17
    k[:, :, 5] = (sign * scale * size[at])[:, None]
    v = torch.randn(keys, 2, d, generator=torch.Generator().manual_seed(1))
    q, k, v = (t.to(dtype) for t in (q, k, v))
    return q, k, v, (q[0, 0, 5].double() * k[:, 0, 5].double()) / math.sqrt(d)


def prompt(gk, q, k, v):
    op = gk.PromptAttention(G=k.shape[1], Hq=q.shape[1], d=q.shape[2], dtype=q.dtype)
    out, lse = op(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, q.shape[0]], **I32), torch.tensor([0, k.shape[0]], **I32),
                  return_lse=True)
    op.status()
    return out.cpu(), lse.double().cpu()


#: size of a bf16 row's largest score from which it is refused
LIMIT = 2.0 ** 30 * math.log(2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("scale", [2.0 ** 7, 2.0 ** 16])
@pytest.mark.parametrize("n,keys", [(300, 300), (3, 5000)])
def test_prompt_logits_of_billions(gk, n, keys, scale, sign, d, dtype):
    # scale 2^7: logits up to 5.4e8, all answered; 2^16: some rows' largest score is beyond what bf16 takes (NaN), while
    # a row within it may see scores far below.  fp32 answers all.
    q, k, v, x = one_channel(n, keys, d, dtype, sign, scale)
    out, lse = prompt(gk, q, k, v)
    beyond = 0
    for i in range(n):
        seen = x[:i + 1 + keys - n]
        if dtype == BF and float(seen.max().abs()) >= LIMIT:
            assert torch.isnan(out[i]).all() and not torch.isfinite(lse[i]).any(), i
            beyond += 1
            continue
        top = (seen == seen.max()).nonzero()[:, 0]
        want = v[top].double().mean(0).repeat_interleave(2, 0)
        # the scale of the weights leaves the quotient's rounding; equal keys share the weight
        assert ((out[i].double() - want).abs() <= 2.0 ** -7 * v[top].double().abs().amax(0).repeat_interleave(2, 0)).all(), i
        assert ((lse[i] - seen.max() - math.log(len(top))).abs() <= 2.0 ** -21 * seen.max().abs()).all(), i
    assert (beyond > 0) == (dtype == BF and scale == 2.0 ** 16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,keys", [(300, 300), (3, 5000)])
def test_prompt_scores_far_below_the_others_count_nothing(gk, n, keys, d):
    # the first keys give scores of -1e11, whole tiles and whole parts of them; the rest are ordinary
    g = torch.Generator().manual_seed(5)
    first = keys - n - 40 if keys > n else 150
    q, k, v = (torch.randn(m, h, d, generator=g) for m, h in ((n, 4), (keys, 2), (keys, 2)))
    k[:, :, 0] = 0
    q[:, :, 0] = 2.0 ** 20
    k[:first, :, 0] = -2.0 ** 20 * (1 + torch.rand(first, 2, generator=g))
    q, k, v = (t.to(BF) for t in (q, k, v))
    out, lse = prompt(gk, q, k, v)
    seen_from = first if keys == n else 0                   # the first rows see nothing else
    want, wlse, tol, ltol = R.prompt(q[seen_from:], k[first:], v[first:], [0, n - seen_from],
                                     [0, keys - first], bf16=True)
    assert ((out[seen_from:].double() - want).abs() <= tol).all()
    assert ((lse[seen_from:] - wlse).abs() <= ltol).all()
    assert torch.isnan(out[:seen_from]).all() and not torch.isfinite(lse[:seen_from]).any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_paged_logits_of_billions(gk, d, dtype):
    B, G, Hq, ps, n = 3, 2, 8, 32, 1000
    table, pages = R.scattered_table(np.random.default_rng(1), np.full((1, B, G), n), ps)
    g = torch.Generator().manual_seed(3)
    K, V = torch.zeros(pages, ps, d).to(dtype), torch.randn(pages, ps, d, generator=g).to(dtype)
    q = torch.zeros(B, Hq, d).to(dtype)
    q[:, :, 5] = 2.0 ** 17
    size = torch.tensor([2.0 ** (i // 128) * (1 + (i % 128) / 128) for i in range(n)])
    want = torch.empty(B, Hq, d, dtype=dtype)
    e = torch.arange(n)
    for b, h in np.ndindex(B, G):
        p = torch.randperm(n, generator=g)
        K[table[0, b, h][e // ps].long(), e % ps, 5] = (2.0 ** 16 * size[p]).to(dtype)
        top = int(p.argmax())
        want[b, h * Hq // G:(h + 1) * Hq // G] = V[int(table[0, b, h, top // ps]), top % ps]
    for lm in (None, torch.zeros(pages, ps, device="cuda")):
        c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.full((1, B, G), n, **I32), log_m=lm, Hq=Hq)
        got = c.attention(0, q.cuda())
        c.status()
        assert torch.equal(got.cpu(), want)
