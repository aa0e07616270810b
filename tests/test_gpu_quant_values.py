"""Decoding attention over quantised pages where large values have little weight: what an entry adds goes by its weight
and its value together."""
import math

import numpy as np
import pytest
import torch

from . import serving_reference as R
from .test_gpu_quant_attention import BF, F32, pages, real

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lm,by", [(torch.finfo(torch.float32).min, 246 - 127), (-1000.0, 100), (-40.0, 50), (-40.0, 58), (-25.0, 20),
                                   (-80.0, 110)])
@pytest.mark.parametrize("every", [5, 97])
def test_large_values_of_little_weight(gk, dtype, d, lm, by, every):
    lens = np.array([[[700, 130], [3, 5000]]])
    table, n = R.scattered_table(np.random.default_rng(1), lens, 16)
    ((K, ks), (V, vs)), m = pages(2, n, 16, d, spread=1.0)
    vs.view(-1)[every // 2::every] = 127 + by - 8              # largest values of about 2^by
    m.view(-1)[every // 2::every] = lm
    q = torch.randn(2, 8, d, generator=torch.Generator().manual_seed(3)).to(dtype)
    lens_t = torch.from_numpy(lens.astype(np.int32))
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), lens_t.cuda(), log_m=m.cuda(), Hq=8, k_scale=ks.cuda(), v_scale=vs.cuda(),
                      dtype=dtype)
    out = c.attention(0, q.cuda()).double().cpu()
    c.status()
    Kr, Vr = real(K, ks), real(V, vs)
    for b, g in np.ndindex(2, 2):
        k, v = (R.entries(t, table[0, b, g], int(lens[0, b, g])).double() for t in (Kr, Vr))
        bias = R.entries(m, table[0, b, g], int(lens[0, b, g])).double()
        qq = q[b, g * 4:g * 4 + 4].double()
        want, _, w = R.attend(qq, k, v, bias=bias)
        sure = w @ v.abs()
        # relative errors of the weights (16 bits; their logits', with that of adding log m) and of n fp32 sums, each of
        # sum w |v|; the output's rounding
        dx = R.logit_error(qq, k, len(k)) + 2.0 ** -22 * (abs(lm) if abs(lm) < 1e4 else 8)
        tol = sure * (2.0 ** -(16 if dtype == BF else 24) + 2 * dx + 2.0 ** -24 * (len(k) + 64))
        tol = tol + 2.0 ** -(8 if dtype == BF else 24) * want.abs() * 1.01 + 1e-30
        got = out[b, g * 4:g * 4 + 4]
        assert torch.isfinite(got).all()
        assert ((got - want).abs() <= tol).all(), f"{float(((got - want).abs() / tol).max()):.3e} of its bound"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lm", [torch.finfo(torch.float32).min, -1e30, -1e9, 3e6, 1e9])
@pytest.mark.parametrize("by", [-90, -30, 30, 100])
def test_values_beside_large_log_m(gk, dtype, lm, by):
    # every entry as large a log m: equal weights, whatever the values' scales
    lens = np.array([[[700, 130]]])
    table, n = R.scattered_table(np.random.default_rng(4), lens, 16)
    ((K, ks), (V, vs)), m = pages(5, n, 16, 64, spread=4.0)
    K.view(torch.uint8).fill_(0)
    vs.copy_((vs.int() + by).clamp(7, 246).to(torch.uint8))
    m.fill_(lm)
    q = torch.randn(1, 8, 64, generator=torch.Generator().manual_seed(6)).to(dtype)
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), log_m=m.cuda(), Hq=8,
                      k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype)
    out = c.attention(0, q.cuda()).double().cpu()
    c.status()
    for g in range(2):
        v = R.entries(real(V, vs), table[0, 0, g], int(lens[0, 0, g])).double()
        want, sure = v.mean(0), v.abs().mean(0)
        tol = sure * (2.0 ** -16 + 2.0 ** -24 * (len(v) + 64)) + 2.0 ** -(8 if dtype == BF else 24) * want.abs() * 1.01
        got = out[0, g * 4:g * 4 + 4]
        assert torch.isfinite(got).all() and ((got - want).abs() <= tol).all()
