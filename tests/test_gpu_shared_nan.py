"""NaN codes in quantised shared prefixes reach what they reach in gracekv_quant_attention, wherever in a tile they are."""
import math

import numpy as np
import pytest
import torch

from . import serving_reference as R
from .test_gpu_quant_attention import junk, pages, real
from .test_gpu_shared import BF, F32, KINDS, queries
from .test_gpu_shared_scales import Side, no_zeros

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("n", [256, 300])
def test_nan_codes_without_weight(gk, dtype, B, n):
    # log m = -inf takes the weight away but leaves a NaN what it is, in a full tile and in one with entries that are not
    # there: a NaN key its head's outputs, a NaN value its channel's; NaN past the length reaches nothing
    lens = np.array([[[n, n]]])
    table, count = R.scattered_table(np.random.default_rng(8), lens, 16)
    for at in (n - 3, 7):
        ((K, ks), (V, vs)), lm = pages(9, count, 16, 64)
        out_of = junk(table, lens, 16, count)
        for t in (K, V):
            t.view(torch.uint8)[out_of] = 0x7f
        K.view(torch.uint8)[table[0, 0, 0, at // 16], at % 16, 9] = 0x7f
        V.view(torch.uint8)[table[0, 0, 1, at // 16], at % 16, 11] = 0xff
        for h in range(2):
            lm[table[0, 0, h, at // 16], at % 16] = -math.inf
        prefix = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), Hq=4,
                               log_m=lm.cuda(), k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype)
        own = Side(gk, np.full((1, B, 2), 9), 16, 4, 64, dtype, 10, lambda *a: None)
        f = gk.SharedAttention(own.cache, prefix)
        q = queries(B, 4, 64, dtype, 11)
        out = f(0, q.cuda()).cpu()
        f.status()
        keep = torch.arange(64) != 11
        assert torch.isnan(out[:, :2]).all() and torch.isnan(out[:, 2:, 11]).all() and torch.isfinite(out[:, 2:, keep]).all()
        # as over the same entries as one request's own
        alone = prefix.attention(0, q[:1].cuda()).cpu()
        assert torch.equal(torch.isnan(alone), torch.isnan(out[:1]))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan_in_quantised_prefixes(gk, dtype):
    # a NaN key of a prefix reaches its head's requests, of a request's own itself alone; a NaN value its channel
    a = Side(gk, np.full((1, 4, 2), 20), 16, 4, 64, dtype, 1, lambda *x: None)
    p = Side(gk, np.full((1, 2, 2), 300), 16, 4, 64, dtype, 2, lambda *x: None)
    q = queries(4, 4, 64, dtype, 3)
    q[3, 3, 7] = math.inf
    byte = torch.uint8
    p.cache.K.view(byte)[p.table[0, 0, 0, 5], 3, 9] = 0x7f
    p.cache.V.view(byte)[p.table[0, 1, 1, 18], 2, 11] = 0x7f
    a.cache.K.view(byte)[a.table[0, 2, 0, 1], 1, 1] = 0xff
    f = gk.SharedAttention(a.cache, p.cache)
    out = f(0, q.cuda(), cu_prefix=torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")).cpu()
    f.status()
    assert torch.isnan(out[:2, :2]).all() and torch.isfinite(out[:2, 2:]).all()
    assert torch.isnan(out[2, :2]).all() and torch.isfinite(out[3, :2]).all()
    assert torch.isnan(out[2:, 2:, 11]).all() and torch.isnan(out[3, 3]).all()
    keep = torch.arange(64) != 11
    assert torch.isfinite(out[2, 2:, keep]).all() and torch.isfinite(out[3, 2, keep]).all()


@pytest.mark.parametrize("dtype,quant,wide", [(*k, False) for k in KINDS] + [(BF, True, True), (F32, True, True)])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("lm", [math.nan, math.inf])
def test_log_m_that_is_no_number(gk, dtype, quant, wide, B, lm):
    # in a prefix it makes its head NaN for all requests, in a request's own entries for that one; with keys of scales close
    # together and far apart, and whatever its page neighbours hold
    lens = np.array([[[300, 300]]])
    table, count = R.scattered_table(np.random.default_rng(12), lens, 16)
    ((K, ks), (V, vs)), m = pages(13, count, 16, 64)
    no_zeros(K, ks, V, vs, m)
    if wide:
        ks.view(-1)[::50] = 80
    for at in (299, 20):
        g = torch.Generator().manual_seed(at)
        own_m = torch.rand(B * 2, 16, generator=g)
        own_m[2 * (B - 1) + 1, 3] = lm
        pre_m = m.clone()
        pre_m[table[0, 0, 0, at // 16], at % 16] = lm
        sc = dict(k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype) if quant else {}
        Kp, Vp = (K, V) if quant else (real(K, ks).to(dtype), real(V, vs).to(dtype))
        i32 = dict(dtype=torch.int32, device="cuda")
        prefix = gk.PagedCache(Kp.cuda(), Vp.cuda(), table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), Hq=4,
                               log_m=pre_m.cuda(), **sc)
        x = torch.randn(2, B * 2, 16, 64, generator=g).to(dtype).cuda()
        own = gk.PagedCache(x[0], x[1], torch.arange(B * 2, **i32).view(1, B, 2, 1), torch.full((1, B, 2), 9, **i32), Hq=4,
                            log_m=own_m.cuda())
        f = gk.SharedAttention(own, prefix)
        out = f(0, queries(B, 4, 64, dtype, 14).cuda()).cpu()
        f.status()
        assert torch.isnan(out[:, :2]).all() and torch.isfinite(out[:B - 1, 2:]).all() and torch.isnan(out[B - 1, 2:]).all()
