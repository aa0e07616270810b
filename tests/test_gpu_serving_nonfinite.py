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
