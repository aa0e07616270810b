"""The quantised cache's calls without a GPU: every argument check returns its
status before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from . import quant_reference as Q
from .test_serving_host import BF, Tensor
from .test_serving_abi import P, gk, paged  # noqa: F401


def calls(gk, c, scales=(P, P)):
    L = gk.lib()
    sc = None if scales is None else C.byref(gk.GkvPagedScales(*scales))
    tokens = lambda N=3, cu=P, pos=P, k=(P, 128, 64), v=(P, 128, 64), q=(P, 512, 64), o=(P, 512, 64): C.byref(  # noqa: E731
        gk.GkvPagedTokens(N, cu, pos, k[0], v[0], q[0], o[0], *k[1:], *v[1:], *q[1:], *o[1:]))
    return {
        "load": lambda b=0, K=P, V=P, m=P, off=P, E=5, ws=P: L.gracekv_quant_load(c, sc, b, K, V, m, off, E, ws, None),
        "append": lambda l=0, ws=P, **kw: L.gracekv_quant_append(c, sc, l, tokens(**kw), ws, None),
        "read": lambda l=0, N=3, cu=P, k=(P, 128, 64), v=(P, 128, 64), ws=P: L.gracekv_paged_read(
            c, sc, l, C.byref(gk.GkvPagedRows(N, cu, k[0], v[0], *k[1:], *v[1:])), ws, None),
        "unload": lambda b=0, K=P, V=P, m=P, off=P, E=5, ws=P: L.gracekv_paged_unload(c, sc, b, K, V, m, off, E, ws, None),
    }


@pytest.mark.parametrize("kw,status", [
    (dict(L=0), 1), (dict(G=0), 1), (dict(Hq=3), 1), (dict(dtype=7), 1), (dict(d=80), 8), (dict(Hq=32), 8), (dict(page_size=0), 1),
    (dict(n_pages=1 << 31), 1), (dict(K=None), 1), (dict(V=P + 8), 1), (dict(table=None), 1), (dict(lens=P + 1), 1),
])
def test_cache_refusals(gk, kw, status):  # noqa: F811
    for name, call in calls(gk, paged(gk, **kw)).items():
        assert call() == status, name
    for name, call in calls(gk, None).items():
        assert call() == gk.GKV_EINVAL, name


@pytest.mark.parametrize("scales", [(None, P), (P, None), (P + 8, P), (P, P + 4)])
def test_scales_refusals(gk, scales):  # noqa: F811
    for name, call in calls(gk, paged(gk), scales).items():
        assert call() == gk.GKV_EINVAL, name


def test_call_refusals(gk):  # noqa: F811
    c = calls(gk, paged(gk))
    none = calls(gk, paged(gk), None)
    for name in ("load", "append"):           # the calls of quantised pages need their scales
        assert none[name]() == gk.GKV_EINVAL
    for kw in (dict(b=3), dict(b=-1), dict(K=None), dict(V=P + 4), dict(off=None), dict(off=P + 4), dict(E=-1), dict(E=1 << 31),
               dict(ws=None), dict(m=P + 1), dict(ws=P + 64)):
        assert c["load"](**kw) == gk.GKV_EINVAL, kw
        for x in (c, none):
            assert x["unload"](**kw) == gk.GKV_EINVAL, kw
    for kw in (dict(l=2), dict(l=-1), dict(N=-1), dict(cu=None, N=2), dict(cu=P + 2), dict(pos=None), dict(k=(None, 128, 64)),
               dict(v=(P, 130, 64)), dict(q=(P, 512, 4)), dict(o=(None, 0, 0)), dict(o=(P, 512, 8)), dict(ws=None)):
        assert c["append"](**kw) == gk.GKV_EINVAL, kw
    for kw in (dict(l=2), dict(l=-1), dict(N=-1), dict(cu=None, N=2), dict(cu=P + 2), dict(k=(None, 128, 64)), dict(v=(P, 130, 64)),
               dict(k=(P + 8, 128, 64)), dict(k=(P, 0, 64)), dict(v=(P, 128, 8)), dict(k=(P, -128, 64)), dict(ws=None), dict(ws=P + 16)):
        for x in (c, none):
            assert x["read"](**kw) == gk.GKV_EINVAL, kw
    assert gk.lib().gracekv_paged_read(paged(gk), None, 0, None, P, None) == gk.GKV_EINVAL
    assert c["append"](N=0) == gk.GKV_OK and c["read"](N=0) == gk.GKV_OK          # nothing to do: nothing is launched
    for base in (-1.0, 0.5, float("nan"), float("inf")):
        assert calls(gk, paged(gk, rope_base=base))["append"]() == gk.GKV_EINVAL
    assert calls(gk, paged(gk, log_m=None))["load"]() == gk.GKV_EINVAL


def test_objects_refuse_other_types(monkeypatch, gk):  # noqa: F811
    u8, i32, e4 = dict(dtype=torch.uint8), dict(dtype=torch.int32), dict(dtype=torch.float8_e4m3fn)
    table, lens = Tensor(1, 3, 2, 2, **i32), Tensor(1, 3, 2, **i32)

    def make(K, V, **kw):
        return gk.PagedCache(K, V, table, lens, Hq=4, **kw)

    plain, codes, scale = Tensor(4, 16, 64), Tensor(4, 16, 64, **e4), Tensor(4, 16, **u8)
    for args, kw in (((codes, codes), {}), ((codes, codes), dict(k_scale=scale)), ((codes, codes), dict(v_scale=scale)),
                     ((plain, plain), dict(k_scale=scale, v_scale=scale)), ((plain, plain), dict(dtype=torch.float32)),
                     ((codes, codes), dict(k_scale=scale, v_scale=scale, dtype=torch.float16)),
                     ((codes, plain), dict(k_scale=scale, v_scale=scale)),
                     ((codes, codes), dict(k_scale=Tensor(4, 15, **u8), v_scale=scale)),
                     ((codes, codes), dict(k_scale=Tensor(4, 16), v_scale=scale)),
                     ((Tensor(4, 16, 64, dtype=torch.float8_e5m2),) * 2, dict(k_scale=scale, v_scale=scale))):
        with pytest.raises(gk.GraceKVError) as e:
            make(*args, **kw)
        assert e.value.status == gk.GKV_EINVAL


def test_the_reference_rounds_as_torch_does():
    # the tests' own rounding against the type's conversion
    x = torch.randn(200, 64) * torch.exp2(torch.randint(-12, 12, (200, 1)).float())
    v, e = Q.quantised(x.double().numpy())
    codes = (x.double() / 2.0 ** torch.from_numpy(e).double()).float().to(torch.float8_e4m3fn)
    assert np.array_equal(codes.double().numpy() * 2.0 ** e, v)
    assert (np.abs(x.double().numpy()).max(-1) <= 448 * 2.0 ** e[:, 0]).all() and (np.abs(x.double().numpy()).max(-1) > 224 * 2.0 ** e[:, 0]).all()


def test_attention_refusals(gk):  # noqa: F811
    L = gk.lib()
    sc = C.byref(gk.GkvPagedScales(P, P))
    call = lambda c, l=0, q=P, out=P, ws=P, s=sc: L.gracekv_quant_attention(c, s, l, q, out, ws, None)  # noqa: E731
    for kw in (dict(l=2), dict(l=-1), dict(q=None), dict(q=P + 8), dict(out=None), dict(out=P + 8), dict(ws=None), dict(ws=P + 1),
               dict(s=None), dict(s=C.byref(gk.GkvPagedScales(P, P + 1)))):
        assert call(paged(gk), **kw) == gk.GKV_EINVAL, kw
    assert call(paged(gk, page_size=24)) == gk.GKV_EUNSUPPORTED and call(None) == gk.GKV_EINVAL


def shared(gk, c=None, p=None, sc=None, psc=None, l=0, cu=P, q=P, out=P, ws=P):
    c, p = paged(gk) if c is None else c, paged(gk) if p is None else p
    return gk.lib().gracekv_shared_attention(c, sc, p, psc, l, cu, q, out, ws, None)


def test_shared_refusals(gk):  # noqa: F811
    for kw in (dict(l=2), dict(l=-1), dict(cu=P + 2), dict(cu=None), dict(q=None), dict(q=P + 8), dict(out=None), dict(out=P + 4),
               dict(ws=None), dict(ws=P + 128), dict(sc=C.byref(gk.GkvPagedScales(P, None))),
               dict(psc=C.byref(gk.GkvPagedScales(P + 2, P)))):
        assert shared(gk, **kw) == gk.GKV_EINVAL, kw
    for kw in (dict(L=1), dict(G=1), dict(Hq=4), dict(d=128), dict(dtype=gk.GKV_F32)):       # caches of different models
        assert shared(gk, p=paged(gk, **kw)) == gk.GKV_EINVAL, kw
        assert shared(gk, c=paged(gk, **kw)) == gk.GKV_EINVAL, kw
    for kw in (dict(B=0), dict(K=None), dict(lens=P + 1), dict(n_pages=0)):
        assert shared(gk, p=paged(gk, **kw)) == gk.GKV_EINVAL and shared(gk, c=paged(gk, **kw)) == gk.GKV_EINVAL, kw
    assert shared(gk, p=paged(gk, page_size=24)) == gk.GKV_EUNSUPPORTED and shared(gk, c=paged(gk, page_size=8)) == gk.GKV_EUNSUPPORTED
    n, L = C.c_size_t(), gk.lib()
    assert L.gracekv_shared_workspace_size(paged(gk), paged(gk, B=1), C.byref(n)) == gk.GKV_OK and n.value > 256
    assert L.gracekv_shared_workspace_size(paged(gk), paged(gk), None) == gk.GKV_EINVAL
    assert L.gracekv_shared_workspace_size(None, paged(gk), C.byref(n)) == gk.GKV_EINVAL
    assert L.gracekv_shared_workspace_size(paged(gk), None, C.byref(n)) == gk.GKV_EINVAL
    assert L.gracekv_shared_workspace_size(paged(gk, d=96), paged(gk, d=96), C.byref(n)) == gk.GKV_EUNSUPPORTED
    assert L.gracekv_shared_status(None, None) == gk.GKV_EINVAL
