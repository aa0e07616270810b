"""A request leaves a cache without log m and comes back: its zeros for log m stay behind."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


@pytest.mark.parametrize("quant", [False, True])
def test_unload_and_load_without_log_m(gk, quant):
    c = gk.PagedCache.allocate(L=1, B=2, G=2, Hq=2, d=64, dtype=torch.bfloat16, n_pages=8, max_pages=2, page_size=16, log_m=False,
                               quantised=quant)
    K, V = (torch.randn(37, 64, device="cuda").bfloat16() for _ in range(2))
    off = torch.tensor([0, 20, 37], device="cuda")
    c.load(0, gk.Cache(K, V, None, torch.zeros(37, device="cuda"), None, None, off), 37)
    k, v, m, o = c.unload_packed(0, 37)
    assert (m == 0).all() and torch.equal(o, off)
    with pytest.raises(gk.GraceKVError) as e:
        c.load_packed(0, k, v, m, o)
    assert e.value.status == gk.GKV_EINVAL
    c.load_packed(0, k, v, None, o)
    again = c.unload_packed(0, 37)
    c.status()
    assert torch.equal(again[0], k) and torch.equal(again[1], v) and torch.equal(again[3], off)
    c.release(0)
    c.load(0, gk.Cache(k, v, None, m, None, None, o), 37)            # load looks at them: none above 0
    assert torch.equal(c.unload(0).K, k)
