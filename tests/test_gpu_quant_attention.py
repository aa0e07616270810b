"""Decoding attention over quantised pages (gracekv_quant_attention) against the
definition in 64 bits on what the rows stand for; the tolerances are those of
the attention over plain pages, as codes and scales enter both products exactly."""
import math

import numpy as np
import pytest
import torch

from . import quant_reference as Q
from . import serving_reference as R

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


def pages(seed, n, ps, d, spread=6.0):
    """Values [n, ps, d] of rows of several sizes, their codes and scales, and log m."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i in range(2):
        x = torch.randn(n * ps, d, generator=g)
        if i:
            x *= torch.exp2(spread * (2 * torch.rand(n * ps, 1, generator=g) - 1))
        x[::11] = 0
        out.append(Q.pool(x))
    lm = torch.log(torch.clamp(torch.exp2(1 + 6 * torch.rand(n, ps, generator=g)) * torch.rand(n, ps, generator=g), min=1.0))
    return [(c.view(n, ps, d), s.view(n, ps)) for c, s in out], lm


def junk(table, lens, ps, n_pages):
    """Pool rows that no sequence holds."""
    held = torch.zeros(n_pages * ps, dtype=torch.bool)
    for i in np.ndindex(*lens.shape):
        e = torch.arange(int(lens[i]))
        held[table[i][e // ps].long() * ps + e % ps] = True
    return ~held.view(n_pages, ps)


def real(codes, scale):
    return torch.from_numpy(Q.values(codes, scale))


def attend(gk, lens, ps, Hq, d, dtype, seed=0, logm=True, l=0, edit=None, q_scale=1.0, finite=True):
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    table, n_pages = R.scattered_table(rng, lens, ps)
    ((K, ks), (V, vs)), lm = pages(seed, n_pages, ps, d)
    if edit:
        edit(K, ks, V, vs, lm)
    kv = real(K, ks), real(V, vs)
    if logm:                                                # without weight: not in the tolerances either
        for t in kv:
            t[lm == -math.inf] = 0
    out_of = junk(table, lens, ps, n_pages)
    for t in (K, V):
        t.view(torch.uint8)[out_of] = 0x7f                  # NaN
    for t in (ks, vs):
        t[out_of] = 255
    lm[out_of] = math.nan
    lens_t = torch.from_numpy(lens.astype(np.int32))
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(lens.shape[1], Hq, d, generator=g)
    q[:, 1::2] *= 3
    q = (q * q_scale).to(dtype)
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), lens_t.cuda(), log_m=lm.cuda() if logm else None, Hq=Hq, k_scale=ks.cuda(),
                      v_scale=vs.cuda(), dtype=dtype)
    out = c.attention(l, q.cuda())
    c.status()
    want, tol = R.decode(q, *kv, lm if logm else None, table, lens_t, l, bf16=dtype == BF)
    got = out.double().cpu()
    if finite:
        assert torch.isfinite(got).all()
        err = (got - want).abs()
        assert (err <= tol).all(), f"{float((err - tol).max()):.3e} over its bound"
        assert (got[want == 0] == 0).all()
    return c, q, out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1025])
def test_lengths(gk, dtype, d, n):
    attend(gk, [[[n, max(0, n - 1)]]], 64, 8, d, dtype, seed=n)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps", [16, 32, 48, 64, 80, 128, 256])
def test_page_sizes(gk, dtype, ps):
    attend(gk, [[[77, 0], [300, 5], [ps, 2 * ps], [ps - 1, ps + 1]]], ps, 4, 128, dtype, seed=ps)
    attend(gk, [[[77, 0], [300, 5], [ps, 2 * ps], [ps - 1, ps + 1]]], ps, 4, 64, dtype, seed=ps, logm=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,G", [(1, 1), (6, 3), (6, 2), (4, 1), (10, 2), (6, 1), (14, 2), (8, 1), (32, 8)])
def test_head_layouts(gk, dtype, Hq, G):
    lens = np.random.default_rng(G).integers(0, 400, (1, 3, G))
    attend(gk, lens, 32, Hq, 128, dtype, seed=Hq)
    attend(gk, lens, 32, Hq, 64, dtype, seed=Hq)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_uneven_and_long(gk, dtype, d):
    # one sequence far longer than the others: split over many CTAs and joined
    attend(gk, [[[40000, 3], [0, 900], [1, 7000]]], 64 if d == 128 else 16, 8, d, dtype, seed=2)


def test_many_sequences_and_layers(gk):
    lens = np.random.default_rng(5).integers(0, 130, (1, 300, 8))
    attend(gk, lens, 32, 32, 64, BF, seed=5)
    lens = np.random.default_rng(7).integers(0, 200, (3, 2, 2))
    for l in range(3):
        attend(gk, lens, 16, 4, 64, BF, seed=7, l=l)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_log_m_extremes(gk, dtype):
    low = torch.finfo(torch.float32).min

    def some(K, ks, V, vs, lm):
        lm[:, ::3] = -math.inf
        lm[:, 1::3] = low

    def none(K, ks, V, vs, lm):
        lm.fill_(-math.inf)

    def lowest(K, ks, V, vs, lm):
        lm.fill_(low)

    for edit in (some, none, lowest):
        _, _, out = attend(gk, [[[90, 200], [1000, 17]]], 16, 8, 128, dtype, seed=8, edit=edit)
    _, _, out = attend(gk, [[[90, 200], [1000, 17]]], 16, 8, 128, dtype, seed=8, edit=none)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scales_of_all_sizes(gk, dtype):
    # keys whose scales reach both ends, with log m = -inf on all but one kind so that the logits stay in range;
    # values 2^-120 to 2^119 beside one another
    def keys(K, ks, V, vs, lm):
        ks.view(-1)[::4] = 7
        ks.view(-1)[1::4] = 246
        lm.view(-1)[1::4] = -math.inf

    attend(gk, [[[90, 203]]], 16, 8, 128, dtype, seed=9, edit=keys, q_scale=2.0 ** -20)

    def values(K, ks, V, vs, lm):
        vs.view(-1)[::3] = 7
        vs.view(-1)[1::3] = 246
        lm.view(-1)[1::3] = -math.inf           # a value of any size without weight
    attend(gk, [[[90, 203]]], 16, 8, 128, dtype, seed=10, edit=values)

    def tiny(K, ks, V, vs, lm):                 # small keys, large queries
        ks.sub_(90)
    attend(gk, [[[90, 203]]], 16, 8, 64, dtype, seed=11, edit=tiny, q_scale=2.0 ** 90)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_small_weights(gk, dtype):
    # one entry of most of the weight, 40000 of 2^-17 each: their sum counts
    def flat(K, ks, V, vs, lm):
        K.view(torch.uint8).fill_(0)
        lm.fill_(-17 * math.log(2))
        lm.view(-1)[5] = 0
        V.view(torch.uint8).fill_(0x38)         # 1
        vs.fill_(127)

    attend(gk, [[[40000, 33]]], 64, 8, 128, dtype, seed=12, edit=flat)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan(gk, dtype):
    # a NaN code of a key: its sequence's heads are NaN; of a value: that channel; NaN or infinite queries: their head
    lens = np.array([[[70, 70], [33, 40]]])
    table, n = R.scattered_table(np.random.default_rng(3), lens, 16)
    ((K, ks), (V, vs)), lm = pages(3, n, 16, 64)
    K.view(torch.uint8)[table[0, 0, 1, 2], 3, 9] = 0xff
    V.view(torch.uint8)[table[0, 1, 0, 1], 2, 5] = 0x7f
    q = torch.randn(2, 4, 64).to(dtype)
    q[0, 0, 7], q[1, 2, 3] = math.nan, math.inf
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), log_m=lm.cuda(), Hq=4,
                      k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype)
    out = c.attention(0, q.cuda()).cpu()
    c.status()
    assert torch.isnan(out[0, 0]).all() and torch.isfinite(out[0, 1]).all()
    assert torch.isnan(out[0, 2:]).all()
    assert torch.isnan(out[1, 2]).all() and torch.isfinite(out[1, 3]).all()
    assert torch.isnan(out[1, :2, 5]).all() and torch.isfinite(out[1, :2, :5]).all() and torch.isfinite(out[1, :2, 6:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_that_are_not_followed(gk, dtype):
    lens = np.array([[[100, 40]]])
    rng = np.random.default_rng(4)
    table, n = R.scattered_table(rng, lens, 16)
    ((K, ks), (V, vs)), lm = pages(4, n, 16, 64)
    q = torch.randn(1, 2, 64).to(dtype)
    bad = table.clone()
    bad[0, 0, 0, 2], bad[0, 0, 1, 0] = n, -5
    lens_t = torch.from_numpy(lens.astype(np.int32))
    c = gk.PagedCache(K.cuda(), V.cuda(), bad.cuda(), lens_t.cuda(), log_m=lm.cuda(), Hq=2, k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype)
    got = c.attention(0, q.cuda())
    with pytest.raises(gk.GraceKVError):
        c.status()
    c.status()
    lm2 = lm.clone()
    lm2[table[0, 0, 0, 2]] = -math.inf
    lm2[table[0, 0, 1, 0]] = -math.inf
    want, tol = R.decode(q, real(K, ks), real(V, vs), lm2, table, lens_t, 0, bf16=dtype == BF)
    assert ((got.double().cpu() - want).abs() <= tol).all()


def test_repeats_streams_and_graphs(gk):
    c, q, out = attend(gk, [[[3000, 40], [0, 700]]], 32, 8, 128, BF, seed=6)
    qd = q.cuda()
    for _ in range(3):
        assert torch.equal(c.attention(0, qd), out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = c.attention(0, qd, stream=s)
    s.synchronize()
    assert torch.equal(got, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        og = c.attention(0, qd)
    c.lens[0, 0, 0] = 9
    g.replay()
    short = c.attention(0, qd)
    assert torch.equal(og, short) and not torch.equal(og, out)
    c.status()


def test_steps_of_a_quantised_cache(gk):
    # load, then advance, append and attention as a server calls them, against the same rows kept in 64 bits
    L, B, G, Hq, d, T = 2, 2, 2, 8, 64, 5
    c = gk.PagedCache.allocate(L=L, B=B, G=G, Hq=Hq, d=d, dtype=BF, n_pages=80, max_pages=8, page_size=16, quantised=True, rope_base=1e4)
    g = torch.Generator().manual_seed(1)
    n = np.array([[30, 45], [17, 60]])
    seqs = {}
    for b in range(B):
        off = np.concatenate([[0], np.cumsum(n.reshape(-1))])
        K, V = (torch.randn(int(off[-1]), d, generator=g).to(BF) for _ in range(2))
        m = torch.rand(int(off[-1]), generator=g) * 3
        c.load(b, gk.Cache(K.cuda(), V.cuda(), None, m.cuda(), None, None, torch.from_numpy(off).cuda()), int(off[-1]))
        for l, h in np.ndindex(L, G):
            a, z = off[l * G + h], off[l * G + h + 1]
            seqs[l, b, h] = [torch.from_numpy(Q.quantised(K[a:z].double().numpy())[0]), torch.from_numpy(Q.quantised(V[a:z].double().numpy())[0]),
                             m[a:z].double()]
    for t in range(T):
        c.advance()
        pos = torch.full((B,), 200 + t, dtype=torch.int32, device="cuda")
        for l in range(L):
            q, k, v = (torch.randn(B, h, d, generator=g).to(BF).cuda() for h in (Hq, G, G))
            qr = c.append(l, k, v, pos, q=q)
            kk, vv = c.read(l, B)
            out = c.attention(l, qr).double().cpu()
            for b, h in np.ndindex(B, G):
                s = seqs[l, b, h]
                s[0], s[1] = torch.cat([s[0], kk[b, h].double().cpu()[None]]), torch.cat([s[1], vv[b, h].double().cpu()[None]])
                s[2] = torch.cat([s[2], torch.zeros(1, dtype=torch.float64)])
                at = slice(h * 4, h * 4 + 4)
                o, _, w = R.attend(qr[b, at].double().cpu(), s[0], s[1], bias=s[2])
                tol = R.attend_bound(qr[b, at].double().cpu(), s[0], s[1], o, w, weight_bits=16, out_bits=8) + 2.0 ** -20 * float(s[1].abs().max())
                assert ((out[b, at] - o).abs() <= tol).all()
    c.status()
