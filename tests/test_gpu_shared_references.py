"""Attention over a shared prefix where logits, or log m, are as large as what masks are held at (2^40, base 2): parts are
joined by their own references, whatever their size, and masks of the lowest or largest log m meet in both caches."""
import math

import pytest
import torch

from . import quant_reference as Q
from .test_gpu_shared import BF, F32, KINDS

pytestmark = pytest.mark.gpu
LOW, TOP = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


class Entries:
    """B sequences of n entries of one KV head: first channels of the keys, log m, values drawn."""

    def __init__(self, gk, first, lm, d, Hq, dtype, quant, seed):
        B, n = first.shape
        pages = -(-n // 16)
        K, V = torch.zeros(B, pages * 16, d), torch.randn(B, pages * 16, d, generator=torch.Generator().manual_seed(seed))
        K[:, :n, 0] = first
        m = torch.zeros(B, pages * 16)
        m[:, :n] = lm
        sc = {}
        shape = (B * pages, 16, d)
        if quant:
            (K, ks), (V, vs) = Q.pool(K.view(-1, d)), Q.pool(V.view(-1, d))
            self.V = torch.from_numpy(Q.values(V, vs)).view(B, -1, d)
            sc = dict(k_scale=ks.view(shape[:2]).cuda(), v_scale=vs.view(shape[:2]).cuda(), dtype=dtype)
        else:
            K, V = K.to(dtype), V.to(dtype)
            self.V = V.double()
        i32 = dict(dtype=torch.int32, device="cuda")
        self.cache = gk.PagedCache(K.view(shape).cuda(), V.view(shape).cuda(), torch.arange(B * pages, **i32).view(1, B, 1, pages),
                                   torch.full((1, B, 1), n, **i32), Hq=Hq, log_m=m.view(shape[:2]).cuda(), **sc)


def outputs(gk, own, prefix, q0, dtype, Hq):
    B, d = own.cache.B, own.cache.d
    q = torch.zeros(B, Hq, d)
    q[..., 0] = q0
    f = gk.SharedAttention(own.cache, prefix.cache)
    out = f(0, q.to(dtype).cuda())
    f.status()
    return out.double().cpu()


def close(got, want, dtype):
    """One weight, or two equal ones: what is left is the rounding of the output, and of an fp32 quotient."""
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= (2.0 ** -8 if dtype == BF else 2.0 ** -22) * want.abs() + 1e-30).all()


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("sign,ratio,size", [(1, 2.0, 20), (-1, 2.0, 20), (1, 1.125, 20), (-1, 1.125, 19), (1, 2.0, 24)])
def test_the_largest_logit_wins_whatever_its_size(gk, dtype, quant, d, B, sign, ratio, size):
    # logits of 2^41 and 2^42 and the like: one entry has all of the weight, in any piece of the prefix or in the own entries
    Hq, n = 4, 3000
    less, more = (2.0 ** size, ratio * 2.0 ** size) if sign > 0 else (-ratio * 2.0 ** size, -2.0 ** size)
    for at in (5, 1700, n - 1, None):
        first, mine = torch.full((1, n), less), torch.full((B, 20), less)
        if at is None:
            mine[:, 7] = more
        else:
            first[0, at] = more
        own = Entries(gk, mine, 0.0, d, Hq, dtype, quant, 1)
        pre = Entries(gk, first, 0.0, d, Hq, dtype, quant, 2)
        got = outputs(gk, own, pre, 2.0 ** 24, dtype, Hq)
        want = own.V[:, 7] if at is None else pre.V[:, at]
        close(got, want[:, None].expand_as(got), dtype)


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("B", [3, 40])
def test_masks_lose_to_any_logit_above_them(gk, dtype, quant, B):
    # one side all of the lowest log m, the other with logits of -2^30
    Hq, n, d = 4, 1500, 64
    for masked in ("prefix", "own"):
        first, mine = torch.full((1, n), -2.0 ** 10), torch.full((B, 20), -2.0 ** 10)
        first[0, 900] = mine[:, 3] = -2.0 ** 9
        own = Entries(gk, mine, LOW if masked == "own" else 0.0, d, Hq, dtype, quant, 3)
        pre = Entries(gk, first, LOW if masked == "prefix" else 0.0, d, Hq, dtype, quant, 4)
        got = outputs(gk, own, pre, 2.0 ** 24, dtype, Hq)
        want = own.V[:, 3] if masked == "prefix" else pre.V[:, 900]
        close(got, want[:, None].expand_as(got), dtype)


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("lm", [LOW, TOP, -1e30, 1e13])
def test_masks_meet_in_both_caches(gk, dtype, quant, B, lm):
    # log m beyond the limit counts as the limit: two such entries, one a side, have half of the weight each, and of the
    # lowest ones every entry as much as any other, with logits that are lost beside it
    Hq, n, d = 4, 1500, 64
    first, mine = torch.full((1, n), 0.25), torch.full((B, 20), -0.5)
    if lm > 0:
        a, b = torch.zeros(1, n), torch.zeros(B, 20)
        a[0, 1111] = b[:, 4] = lm
    else:
        a, b = lm, lm
    own, pre = Entries(gk, mine, b, d, Hq, dtype, quant, 5), Entries(gk, first, a, d, Hq, dtype, quant, 6)
    got = outputs(gk, own, pre, 2.0, dtype, Hq)
    if lm > 0:
        want = (own.V[:, 4] + pre.V[:, 1111]) / 2
        close(got, want[:, None].expand_as(got), dtype)
    else:
        k = n + 20
        want = ((own.V[:, :20].sum(1) + pre.V[:, :n].sum(1)) / k)[:, None].expand_as(got)
        size = float(pre.V.abs().max())
        # equal weights 1 / k: k fp32 sums of values below `size`, and the output's rounding
        assert ((got - want).abs() <= (2.0 ** -8 if dtype == BF else 2.0 ** -22) * want.abs() + 2.0 ** -24 * (k + 64) * size).all()
