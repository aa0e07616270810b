"""Non-finite values that a sequence of the paged cache holds itself: they come
out as the definition has them (a NaN logit is a NaN output, never a zero), and
what does not read them stays bit for bit as it was."""
import math

import numpy as np
import pytest
import torch

from . import serving_reference as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device="cuda")
B, G, HQ, PS = 3, 2, 8, 32
#: every sequence whole; one sequence in many pieces, joined
LENS = {"whole": [[40, 77], [1, 300], [64, 0]], "split": [[9000, 77], [1, 2500], [64, 0]]}


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


def cache(lens, d, dtype, seed=0):
    lens = np.asarray([lens])
    table, pages = R.scattered_table(np.random.default_rng(seed), lens, PS)
    g = torch.Generator().manual_seed(seed)
    K, V = (torch.randn(pages, PS, d, generator=g).to(dtype) for _ in range(2))
    lm = torch.rand(pages, PS, generator=g)
    q = torch.randn(B, HQ, d, generator=g).to(dtype)
    return dict(K=K, V=V, log_m=lm, q=q, table=table, lens=torch.from_numpy(lens.astype(np.int32)))


def attend(gk, s):
    c = gk.PagedCache(s["K"].cuda(), s["V"].cuda(), s["table"].cuda(), s["lens"].cuda(), log_m=s["log_m"].cuda(), Hq=HQ)
    out = c.attention(0, s["q"].cuda()).cpu()
    c.status()
    return out


def row_of(s, b, g, e):
    return int(s["table"][0, b, g, e // PS]), e % PS


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", ["whole", "split"])
def test_paged_attention_keeps_what_is_not_a_number(gk, shape, d, dtype):
    clean = attend(gk, cache(LENS[shape], d, dtype))
    assert torch.isfinite(clean).all()
    n = LENS[shape][0][0]
    group = [(0, h) for h in range(HQ // G)]                 # the query heads of request 0's first KV head
    for e in (0, n // 2, n - 1):
        for what in ("key", "key inf", "log m", "log m inf"):
            s = cache(LENS[shape], d, dtype)
            at = row_of(s, 0, 0, e)
            if what == "key":
                s["K"][at][3] = math.nan
            elif what == "key inf":                          # a logit of +inf
                s["q"][0] = s["q"][0].abs()
                s["K"][at][5] = math.inf
            elif what == "log m":
                s["log_m"][at] = math.nan
            else:
                s["log_m"][at] = math.inf
            base = clean if what != "key inf" else attend(gk, cache(LENS[shape], d, dtype) | dict(q=s["q"]))
            got = attend(gk, s)
            for b in range(B):
                for h in range(HQ):
                    if (b, h) in group:
                        assert torch.isnan(got[b, h]).all(), (what, e, b, h)
                    else:
                        assert torch.equal(got[b, h], base[b, h]), (what, e, b, h)
    # a query: its own head alone
    s = cache(LENS[shape], d, dtype)
    s["q"][0, 2, 7] = math.nan
    got = attend(gk, s)
    assert torch.isnan(got[0, 2]).all()
    got[0, 2] = clean[0, 2]
    assert torch.equal(got, clean)
    # a sequence that holds nothing gives 0 whatever its query
    s = cache(LENS[shape], d, dtype)
    s["q"][2] = math.nan
    got = attend(gk, s)
    assert (got[2, HQ // G:] == 0).all() and torch.isnan(got[2, :HQ // G]).all() and torch.equal(got[:2], clean[:2])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", ["whole", "split"])
def test_paged_attention_of_the_largest_log_m(gk, shape, dtype):
    # finite as it is: one entry of it takes all the weight, entries of nothing else share it
    top = torch.finfo(torch.float32).max
    s = cache(LENS[shape], 128, dtype)
    at = row_of(s, 0, 0, 17)
    s["log_m"][at] = top
    assert torch.equal(attend(gk, s)[0, :HQ // G], s["V"][at].expand(HQ // G, -1))
    s["log_m"].fill_(top)
    want, tol = R.decode(s["q"], s["K"], s["V"], s["log_m"], s["table"], s["lens"], 0, bf16=dtype == BF)
    got = attend(gk, s).double()
    # the bound with the logits' size: log m takes them all to one value, so only sums and rounding are left
    assert torch.isfinite(got).all()
    vmax = float(s["V"].abs().max())
    n = max(max(r) for r in LENS[shape])
    bits = R.BITS_BF16 if dtype == BF else R.BITS_F32
    weights = 2.0 ** -16 if dtype == BF else 2.0 ** -24
    assert ((got - want).abs() <= vmax * (2.0 ** -20 + weights + 2.0 ** -24 * (n + 64)) + 2.0 ** -bits * want.abs() * 1.01).all()


# ------------------------------------------------------------------- the prompt's attention
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk", [(300, 300), (5, 4000)])
def test_prompt_attention_keeps_what_is_not_a_number(gk, nq, nk, d, dtype):
    g = torch.Generator().manual_seed(nq)
    q0, k0, v0 = (torch.randn(n, h, d, generator=g).to(dtype) for n, h in ((nq, 8), (nk, 2), (nk, 2)))
    q0 = q0.abs()                                            # an infinite key gives an infinite logit of its sign
    op = gk.PromptAttention(G=2, Hq=8, d=d, dtype=dtype)
    cq, ck = torch.tensor([0, nq], **I32), torch.tensor([0, nk], **I32)

    def run(q=q0, k=k0, v=v0):
        out, lse = op(q.cuda(), k.cuda(), v.cuda(), cq, ck, return_lse=True)
        op.status()
        return out.cpu(), lse.cpu()

    clean, lclean = run()
    assert torch.isfinite(clean.float()).all()
    # a query: its own row and head alone
    q = q0.clone()
    q[3, 5, 7] = math.nan
    out, lse = run(q=q)
    assert torch.isnan(out[3, 5]).all() and torch.isnan(lse[3, 5])
    out[3, 5], lse[3, 5] = clean[3, 5], lclean[3, 5]
    assert torch.equal(out, clean) and torch.equal(lse, lclean)
    for e in (0, nk - nq + 2, nk - 1, nk // 2):
        first = max(0, e - (nk - nq))                        # the first query that sees key e
        for value in (math.nan, math.inf):
            k = k0.clone()
            k[e, 1, 9] = value
            out, lse = run(k=k)
            assert torch.isnan(out[first:, 4:]).all() and not torch.isfinite(lse[first:, 4:]).any()
            assert torch.equal(out[:, :4], clean[:, :4]) and torch.equal(out[:first], clean[:first])
            assert torch.equal(lse[:, :4], lclean[:, :4]) and torch.equal(lse[:first], lclean[:first])
        # a logit of -inf weighs nothing, as one that is merely far below the others
        k, far = k0.clone(), k0.clone()
        k[e, 1, 9], far[e, 1, 9] = -math.inf, -1e30
        if e > 0:
            a, b = run(k=k), run(k=far)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        # a value: its channel alone, in every query that sees it
        v = v0.clone()
        v[e, 0, 2] = math.nan
        out, lse = run(v=v)
        assert torch.isnan(out[first:, :4, 2]).all() and torch.equal(lse, lclean)
        out[..., :4, 2] = clean[..., :4, 2]
        assert torch.equal(out, clean)
    # all logits -inf: no weight at all
    out, lse = run(k=torch.full_like(k0, -math.inf))
    assert (out == 0).all() and torch.isinf(lse).all() and (lse < 0).all()
