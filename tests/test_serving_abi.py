"""Serving calls of the C ABI without a GPU: every argument check returns its
status before anything is launched."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def gk():
    from paper_2608_07001_gb300 import build_ext
    build_ext.build()
    from paper_2608_07001_gb300 import gracekv
    gracekv.lib()
    return gracekv


P = 1 << 20       # stands for an aligned device pointer; nothing reads it


def prompt(gk, **kw):
    a = dict(G=2, Hq=8, d=128, dtype=gk.GKV_BF16, n_seqs=1, n_q=4, n_k=4, cu_q=P, cu_k=P, q=P, k=P, v=P, out=P, lse=P,
             q_ts=1024, q_hs=128, k_ts=256, k_hs=128, v_ts=256, v_hs=128, o_ts=1024, o_hs=128)
    a.update(kw)
    return C.byref(gk.GkvPrompt(**a))


@pytest.mark.parametrize("kw,status", [
    (dict(G=0), 1), (dict(Hq=7), 1), (dict(dtype=2), 1), (dict(n_q=-1), 1), (dict(n_k=1 << 31), 1), (dict(n_seqs=-1), 1),
    (dict(cu_q=None), 1), (dict(cu_k=P + 2), 1), (dict(q=None), 1), (dict(k=P + 8), 1), (dict(v=None), 1), (dict(out=P + 4), 1),
    (dict(lse=P + 1), 1), (dict(q_ts=1020), 1), (dict(k_hs=-128), 1), (dict(v_ts=4), 1), (dict(o_hs=2), 1),
    (dict(dtype=0, q_ts=1022), 1), (dict(d=96), 8), (dict(d=256), 8), (dict(G=1, Hq=9), 8), (dict(n_q=1 << 40), 1),
])
def test_prompt_refusals(gk, kw, status):
    assert gk.lib().gracekv_prompt_attention(prompt(gk, **kw), P, None) == status


def test_prompt_workspace(gk):
    L, n = gk.lib(), C.c_size_t()
    assert L.gracekv_prompt_attention(None, P, None) == gk.GKV_EINVAL
    assert L.gracekv_prompt_attention(prompt(gk), None, None) == gk.GKV_EINVAL
    assert L.gracekv_prompt_attention(prompt(gk), P + 16, None) == gk.GKV_EINVAL
    assert L.gracekv_prompt_workspace_size(prompt(gk), C.byref(n)) == gk.GKV_OK and n.value >= 256
    assert L.gracekv_prompt_workspace_size(prompt(gk), None) == gk.GKV_EINVAL
    assert L.gracekv_prompt_workspace_size(prompt(gk, d=32), C.byref(n)) == gk.GKV_EUNSUPPORTED
    assert L.gracekv_prompt_status(None, None) == gk.GKV_EINVAL
    # nothing to do is no error and launches nothing
    assert L.gracekv_prompt_attention(prompt(gk, n_seqs=0), P, None) == gk.GKV_OK
    assert L.gracekv_prompt_attention(prompt(gk, n_q=0, q=None, out=None), P, None) == gk.GKV_OK


def paged(gk, **kw):
    a = dict(L=2, B=3, G=2, Hq=8, d=64, dtype=gk.GKV_BF16, page_size=16, max_pages=4, n_pages=10, K=P, V=P, log_m=P, table=P,
             lens=P, rope_base=1e4)
    a.update(kw)
    return C.byref(gk.GkvPagedCache(**a))


def calls(gk, c):
    L = gk.lib()
    yield "load", lambda b=0, K=P, V=P, m=P, off=P, E=5, ws=P: L.gracekv_paged_load(c, b, K, V, m, off, E, ws, None)
    yield "append", lambda l=0, N=3, cu=P, pos=P, k=(P, 128, 64), v=(P, 128, 64), q=(P, 512, 64), o=(P, 512, 64), ws=P: \
        L.gracekv_paged_append(c, l, C.byref(gk.GkvPagedTokens(N, cu, pos, k[0], v[0], q[0], o[0], *k[1:], *v[1:], *q[1:], *o[1:])),
                               ws, None)
    yield "attention", lambda l=0, q=P, out=P, ws=P: L.gracekv_paged_attention(c, l, q, out, ws, None)
    yield "advance", lambda cu=P: L.gracekv_paged_advance(c, cu, None)


@pytest.mark.parametrize("kw,status", [
    (dict(L=0), 1), (dict(B=0), 1), (dict(G=0), 1), (dict(Hq=3), 1), (dict(dtype=7), 1), (dict(d=80), 8), (dict(Hq=32), 8),
    (dict(page_size=0), 1), (dict(max_pages=0), 1), (dict(n_pages=0), 1), (dict(n_pages=1 << 31), 1), (dict(K=None), 1),
    (dict(V=P + 8), 1), (dict(log_m=P + 2), 1), (dict(table=None), 1), (dict(lens=P + 1), 1),
    (dict(page_size=1 << 20, max_pages=1 << 12), 1),
])
def test_paged_cache_refusals(gk, kw, status):
    for name, call in calls(gk, paged(gk, **kw)):
        assert call() == status, name
    for name, call in calls(gk, None):
        assert call() == gk.GKV_EINVAL, name


def test_paged_call_refusals(gk):
    c = dict(calls(gk, paged(gk)))
    for kw in (dict(b=3), dict(b=-1), dict(K=None), dict(V=P + 4), dict(off=None), dict(off=P + 4), dict(E=-1), dict(E=1 << 31),
               dict(ws=None), dict(m=P + 1), dict(ws=P + 64)):
        assert c["load"](**kw) == gk.GKV_EINVAL, kw
    for kw in (dict(l=2), dict(l=-1), dict(N=-1), dict(cu=None, N=2), dict(cu=P + 2), dict(pos=None), dict(k=(None, 128, 64)),
               dict(v=(P, 130, 64)), dict(q=(P, 512, 4)), dict(o=(None, 0, 0)), dict(q=(None, 0, 0)), dict(k=(P, -128, 64)),
               dict(ws=None), dict(pos=P + 1)):
        assert c["append"](**kw) == gk.GKV_EINVAL, kw
    for kw in (dict(l=2), dict(l=-1), dict(q=None), dict(out=P + 8), dict(ws=P + 1)):
        assert c["attention"](**kw) == gk.GKV_EINVAL, kw
    assert c["advance"](cu=P + 1) == gk.GKV_EINVAL
    assert dict(calls(gk, paged(gk, log_m=None)))["load"]() == gk.GKV_EINVAL          # log m, and nowhere to keep it
    assert dict(calls(gk, paged(gk, page_size=24)))["attention"]() == gk.GKV_EUNSUPPORTED
    for base in (-1.0, 0.5, float("nan"), float("inf")):
        assert dict(calls(gk, paged(gk, rope_base=base)))["append"]() == gk.GKV_EINVAL
    assert gk.lib().gracekv_paged_append(paged(gk), 0, None, P, None) == gk.GKV_EINVAL
    assert c["append"](N=0) == gk.GKV_OK                                              # no token: nothing is launched
    n = C.c_size_t()
    assert gk.lib().gracekv_paged_workspace_size(paged(gk), C.byref(n)) == gk.GKV_OK and n.value >= 256
    assert gk.lib().gracekv_paged_workspace_size(paged(gk), None) == gk.GKV_EINVAL
    assert gk.lib().gracekv_paged_status(None, None) == gk.GKV_EINVAL
