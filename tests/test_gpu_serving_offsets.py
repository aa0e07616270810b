"""Offsets of a packed cache that do not fit: the heads that do are loaded all the
same, the others hold nothing, and the call is reported."""
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


def ascending(lens, first=0):
    return [first + int(n) for n in np.concatenate([[0], np.cumsum(lens)])]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L,G,off,cap", [
    (1, 3, [0, 1000, 200, 900], 64),                      # a step back; the next head starts inside the first one
    (1, 4, [0, 50, 20, 20, 60], 64),
    (1, 4, [0, 500, 5000, 500, 900], 64),                 # past the entries, then back
    (1, 4, [0, 500, -3, 500, 900], 64),
    (1, 3, [0, 1000, 200, 900], 20),                      # and a length that the pages do not hold
    (20, 16, "early", 64),                                # more heads than a block has threads
    (20, 16, "late", 64),
])
def test_heads_whose_offsets_fit_are_loaded(gk, L, G, off, cap, dtype):
    ps, d, b, E = 16, 64, 1, 1000
    n_heads = L * G
    if isinstance(off, str):
        off = ascending([3] * n_heads)
        off[5 if off == "early" else n_heads - 5] = 1
        if off[5] != 1:
            off[n_heads - 5] = 1
    lens = [b1 - a1 if 0 <= a1 <= b1 <= E else 0 for a1, b1 in zip(off[:-1], off[1:])]
    cut = [min(n, cap * ps) for n in lens]
    held = np.zeros((L, 2, G), np.int64)
    held[:, b] = np.asarray(cut).reshape(L, G)
    table, pages = R.scattered_table(np.random.default_rng(0), held, ps)
    t = torch.full((L, 2, G, cap), -1, dtype=torch.int32)
    t[..., :table.shape[-1]] = table
    g = torch.Generator().manual_seed(1)
    K, V = (torch.randn(pages, ps, d, generator=g).to(dtype) for _ in range(2))
    lm = torch.rand(pages, ps, generator=g)
    k, v = (torch.randn(E, d, generator=g).to(dtype) for _ in range(2))
    m = torch.rand(E, generator=g)
    c = gk.PagedCache(K.cuda(), V.cuda(), t.cuda(), torch.full((L, 2, G), 9, **I32), log_m=lm.cuda(), Hq=G)
    c.load_packed(b, k.cuda(), v.cuda(), m.cuda(), torch.tensor(off, dtype=torch.int64, device="cuda"))
    with pytest.raises(gk.GraceKVError) as e:
        c.status()
    assert e.value.status == gk.GKV_EINVAL
    for i in range(n_heads):
        for j in range(cut[i]):
            page, row = int(t[i // G, b, i % G, j // ps]), j % ps
            K[page, row], V[page, row], lm[page, row] = k[off[i] + j], v[off[i] + j], m[off[i] + j]
    held[:, 0] = 9
    assert np.array_equal(c.lens.cpu().numpy(), held)
    assert torch.equal(c.K.cpu(), K) and torch.equal(c.V.cpu(), V) and torch.equal(c.log_m.cpu(), lm)
