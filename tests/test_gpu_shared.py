"""Decoding attention of requests that share prefixes (gracekv_shared_*) against
the definition in 64 bits: one softmax over the prefix slot's entries and the
request's own.  For bf16 rows the prefix's weights are rounded to bf16."""
import math

import numpy as np
import pytest
import torch

from . import quant_reference as Q
from . import serving_reference as R
from .test_gpu_quant_attention import junk, pages, real

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


class Side:
    """One cache: its tensors and what its rows stand for."""

    def __init__(self, gk, lens, ps, Hq, d, dtype, quant, logm, seed, edit=None, extra=3):
        lens = np.asarray(lens)
        self.table, n = R.scattered_table(np.random.default_rng(seed), lens, ps, extra)
        ((K, ks), (V, vs)), lm = pages(seed, n, ps, d, spread=2.0)
        if not quant:
            K, V = real(K, ks).to(dtype), real(V, vs).to(dtype)
        if edit:
            edit(K, V, lm)
        self.K, self.V = ((real(K, ks), real(V, vs)) if quant else (K.double(), V.double()))
        self.lm, self.lens = (lm if logm else None), lens
        if logm:                                            # without weight: not in the tolerances either
            self.K, self.V = (t.masked_fill((lm == -math.inf)[..., None], 0.0) for t in (self.K, self.V))
        out_of = junk(self.table, lens, ps, n)
        sc = {}
        if quant:
            for t in (K, V):
                t.view(torch.uint8)[out_of] = 0x7f
            for t in (ks, vs):
                t[out_of] = 255
            sc = dict(k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype)
        else:
            K[out_of], V[out_of] = math.nan, math.inf
        lm = lm.clone()
        lm[out_of] = math.nan
        self.cache = gk.PagedCache(K.cuda(), V.cuda(), self.table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), Hq=Hq,
                                   log_m=lm.cuda() if logm else None, **sc)

    def rows(self, i):
        """Keys, values and log m of sequence i."""
        n = int(self.lens[i])
        k, v = (R.entries(t, self.table[i], n) for t in (self.K, self.V))
        return k, v, torch.zeros(n).double() if self.lm is None else R.entries(self.lm, self.table[i], n).double()


def expected(q, own, prefix, cu, l=0):
    """(out, bound)."""
    B, Hq, d = q.shape
    G = own.lens.shape[2]
    gq, bf16 = Hq // G, q.dtype == BF
    q = q.double().cpu()
    out, tol = torch.zeros(q.shape).double(), torch.zeros(q.shape).double()
    slot = [next((p for p in range(len(cu) - 1) if cu[p] <= b < cu[p + 1]), -1) for b in range(B)]
    for b, g in np.ndindex(B, G):
        parts = [own.rows((l, b, g))] + ([prefix.rows((l, slot[b], g))] if slot[b] >= 0 else [])
        k, v, bias = (torch.cat(x) for x in zip(*parts))
        at = slice(g * gq, (g + 1) * gq)
        o, _, w = R.attend(q[b, at], k, v, bias=bias)
        out[b, at] = o
        t = R.attend_bound(q[b, at], k, v, o, w, weight_bits=R.BITS_BF16 if bf16 else R.BITS_F32, out_bits=R.BITS_BF16 if bf16 else R.BITS_F32)
        if len(k):
            fin = bias[torch.isfinite(bias) & (bias > -1e30)]
            t = t + 2.0 ** -22 * (float(fin.abs().max()) if fin.numel() else 0.0) * float(v.abs().max())
        tol[b, at] = t
    return out, tol


def queries(B, Hq, d, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(B, Hq, d, generator=g)
    q[:, 1::2] *= 3
    return (q * scale).to(dtype)


def attend(gk, own, pre, cu=None, ps=(16, 32), Hq=8, d=128, dtype=BF, quant=(False, False), logm=(True, True), seed=0, l=0, edit=None,
           scale=1.0):
    own, pre = np.asarray(own), np.asarray(pre)
    a = Side(gk, own, ps[0], Hq, d, dtype, quant[0], logm[0], seed, edit=edit)
    p = Side(gk, pre, ps[1], Hq, d, dtype, quant[1], logm[1], seed + 100, edit=edit)
    q = queries(own.shape[1], Hq, d, dtype, seed + 1, scale)
    f = gk.SharedAttention(a.cache, p.cache)
    cud = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")
    out = f(l, q.cuda(), cu_prefix=cud)
    f.status()
    want, tol = expected(q, a, p, [0, own.shape[1]] if cu is None else cu, l)
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    err = (got - want).abs()
    assert (err <= tol).all(), f"{float((err - tol).max()):.3e} over its bound"
    assert (got[want == 0] == 0).all()
    return f, q, out, cud


KINDS = [(BF, False), (BF, True), (F32, False), (F32, True)]


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [0, 1, 17, 64, 127, 128, 129, 300, 1000])
def test_lengths(gk, dtype, quant, d, n):
    rng = np.random.default_rng(n)
    own = rng.integers(0, 40, (1, 3, 2))
    own[0, 1] = 0
    attend(gk, own, [[[n, max(0, n - 5)]]], d=d, dtype=dtype, quant=(quant, quant), seed=n)


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("ps", [16, 32, 48, 64, 80, 128, 256])
def test_page_sizes(gk, dtype, quant, ps):
    own = np.random.default_rng(ps).integers(0, 200, (1, 5, 2))
    attend(gk, own, [[[2 * ps + 3, 700]]], ps=(ps, ps), dtype=dtype, quant=(quant, quant), seed=ps, logm=(False, True))
    attend(gk, own, [[[5 * ps, ps - 1]]], ps=(16, ps), d=64, dtype=dtype, quant=(quant, quant), seed=ps, logm=(True, False))


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("Hq,G", [(1, 1), (6, 3), (6, 2), (4, 1), (10, 2), (6, 1), (14, 2), (8, 1), (32, 8)])
@pytest.mark.parametrize("B", [1, 70])
def test_head_layouts(gk, dtype, quant, Hq, G, B):
    rng = np.random.default_rng(G + B)
    attend(gk, rng.integers(0, 30, (1, B, G)), rng.integers(200, 600, (1, 1, G)), Hq=Hq, d=128 if B == 1 else 64, dtype=dtype,
           quant=(quant, quant), seed=Hq)


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_batches_of_all_sizes(gk, dtype, quant):
    # around a row tile, a block of rows, and several of them
    for B in (15, 16, 17, 31, 32, 33, 63, 64, 65, 130, 200):
        rng = np.random.default_rng(B)
        attend(gk, rng.integers(0, 20, (1, B, 1)), [[[777]]], Hq=8 if B < 100 else 4, d=64, dtype=dtype, quant=(quant, quant), seed=B)


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_groups(gk, dtype, quant, d):
    # slots of no, one and many requests; of no entries; requests of no slot at both ends
    rng = np.random.default_rng(d)
    own = rng.integers(0, 50, (1, 60, 2))
    pre = rng.integers(100, 900, (1, 6, 2))
    pre[0, 2] = 0
    attend(gk, own, pre, cu=[3, 4, 4, 20, 21, 50, 58], d=d, dtype=dtype, quant=(quant, quant), seed=d)


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_long_prefix(gk, dtype, quant):
    attend(gk, [[[5, 70], [0, 0], [300, 1]]], [[[30000, 12345]]], ps=(16, 64), dtype=dtype, quant=(quant, quant), seed=1)
    attend(gk, [[[5, 70], [0, 0], [300, 1]]], [[[20000, 3]]], ps=(16, 16), d=64, dtype=dtype, quant=(quant, quant), seed=2, logm=(False, False))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_own_entries_of_many_pieces(gk, dtype):
    # a request whose own entries are split over CTAs, joined with its prefix
    attend(gk, [[[20000, 40], [7, 9000]]], [[[1500, 300]]], dtype=dtype, seed=3)
    attend(gk, [[[20000, 40], [7, 9000]]], [[[1500, 300]]], dtype=dtype, seed=4, quant=(True, True), d=64)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("quant", [(True, False), (False, True)])
def test_one_side_quantised(gk, dtype, quant):
    attend(gk, [[[50, 7], [0, 20]]], [[[400, 200]]], dtype=dtype, quant=quant, seed=5)


def test_many_slots_and_layers(gk):
    rng = np.random.default_rng(6)
    own, pre = rng.integers(0, 20, (3, 90, 4)), rng.integers(0, 300, (3, 45, 4))
    for l in range(3):
        attend(gk, own, pre, cu=list(range(0, 91, 2)), Hq=4, d=64, seed=7, l=l)
    # more slots than a block of the plan takes at once
    own, pre = rng.integers(0, 5, (1, 1500, 1)), rng.integers(0, 40, (1, 1300, 1))
    attend(gk, own, pre, cu=list(range(100, 1401)), ps=(16, 16), Hq=2, d=64, seed=8)


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_few_of_many_slots(gk, dtype, quant):
    # the workspace has room for more pieces than run at once; blocks of one and of two row tiles share them
    own = np.random.default_rng(9).integers(0, 30, (1, 50, 2))
    pre = np.full((1, 60, 2), 3)
    pre[0, 7], pre[0, 31] = (3000, 5000), (2500, 40)
    cu = [0] * 8 + [41] * 24 + [50] * 29
    attend(gk, own, pre, cu=cu, d=64, dtype=dtype, quant=(quant, quant), seed=9)


@pytest.mark.parametrize("dtype,quant", KINDS)
@pytest.mark.parametrize("Hq", [2, 10, 14, 16])
@pytest.mark.parametrize("d", [64, 128])
def test_many_short_own_sequences(gk, dtype, quant, Hq, d):
    # several sequences a CTA, whole and cut, of up to eight heads
    rng = np.random.default_rng(Hq)
    own = rng.integers(1, 150, (1, 400, 2))
    if Hq == 14:
        own[0, 5] = 3000
    attend(gk, own, [[[70, 0]]], Hq=Hq, d=d, dtype=dtype, quant=(quant, False), seed=Hq)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
def test_long_prefix_of_small_pages(gk, quant, d, B):
    # windows of looked-up boxes turn many times beside tiles of log m
    attend(gk, np.full((1, B, 1), 2), [[[50011]]], ps=(16, 16), Hq=4, d=d, quant=(quant, quant), seed=B)


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_log_m_extremes(gk, dtype, quant):
    low = torch.finfo(torch.float32).min

    def some(K, V, lm):
        lm[:, ::3] = -math.inf
        lm[:, 1::3] = low

    def none(K, V, lm):
        lm.fill_(-math.inf)

    def lowest(K, V, lm):
        lm.fill_(low)

    def growing(K, V, lm):                   # references that have to follow
        lm.copy_(torch.arange(lm.numel()).view(lm.shape).float() * 0.2)

    for edit in (some, lowest, growing):
        attend(gk, [[[90, 200], [0, 17]]], [[[500, 129]]], dtype=dtype, quant=(quant, quant), seed=9, edit=edit)
    _, _, out, _ = attend(gk, [[[90, 200], [0, 17]]], [[[500, 129]]], dtype=dtype, quant=(quant, quant), seed=9, edit=none)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_large_logits(gk, dtype, quant):
    # softmax of a single entry, wherever it is
    attend(gk, [[[40, 10]] * 20], [[[300, 700]]], dtype=dtype, quant=(quant, quant), seed=10, scale=40.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan(gk, dtype):
    # a NaN key of a prefix reaches its head's requests, of a request's own itself alone; a NaN value its channel
    own, pre = np.full((1, 4, 2), 20), np.full((1, 2, 2), 300)
    a = Side(gk, own, 16, 4, 64, dtype, False, True, 1)
    p = Side(gk, pre, 16, 4, 64, dtype, False, True, 2)
    q = queries(4, 4, 64, dtype, 3)
    q[3, 3, 7] = math.inf
    p.cache.K[p.table[0, 0, 0, 5], 3, 9] = math.nan
    p.cache.V[p.table[0, 1, 1, 18], 2, 11] = math.nan
    a.cache.K[a.table[0, 2, 0, 1], 1, 1] = math.nan
    f = gk.SharedAttention(a.cache, p.cache)
    out = f(0, q.cuda(), cu_prefix=torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")).cpu()
    f.status()
    assert torch.isnan(out[:2, :2]).all() and torch.isfinite(out[:2, 2:]).all()
    assert torch.isnan(out[2, :2]).all() and torch.isfinite(out[3, :2]).all()
    assert torch.isnan(out[2:, 2:, 11]).all() and torch.isnan(out[3, 3]).all()
    keep = torch.arange(64) != 11
    assert torch.isfinite(out[2, 2:, keep]).all() and torch.isfinite(out[3, 2, keep]).all()


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_words_and_pages_that_do_not_fit(gk, dtype, quant):
    rng = np.random.default_rng(11)
    own, pre = rng.integers(1, 40, (1, 12, 2)), rng.integers(200, 500, (1, 4, 2))
    a = Side(gk, own, 16, 4, 64, dtype, quant, True, 12)
    p = Side(gk, pre, 32, 4, 64, dtype, quant, True, 13)
    q = queries(12, 4, 64, dtype, 14)
    f = gk.SharedAttention(a.cache, p.cache)

    def check(cu, groups, reported=True):
        out = f(0, q.cuda(), cu_prefix=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        if reported:
            with pytest.raises(gk.GraceKVError) as e:
                f.status()
            assert e.value.status == gk.GKV_EINVAL
        f.status()
        bounds = [b for g in groups for b in g[1:]]
        assert bounds == sorted(bounds)
        cuts, order = [0], []
        for s, lo, hi in groups:                          # gaps are slots without entries
            order += [None, s]
            cuts += [lo, hi]
        cuts.append(12)
        order.append(None)

        class Laid:
            @staticmethod
            def rows(i):
                s = order[i[1]]
                if s is None:
                    return tuple(x[:0] for x in p.rows((0, 0, 0)))
                return p.rows((0, s, i[2]))
        want, tol = expected(q, a, Laid, cuts)
        assert ((out.double().cpu() - want).abs() <= tol).all()

    check([0, 3, 6, 9, 12], [(0, 0, 3), (1, 3, 6), (2, 6, 9), (3, 9, 12)], reported=False)
    check([0, 3, 2, 9, 12], [(0, 0, 3), (3, 9, 12)])      # slot 1 runs backwards, slot 2 begins inside slot 0
    check([-1, 3, 6, 13, 12], [(1, 3, 6)])
    # a page outside the pool: its entries are skipped
    bad = p.table[0, 1, 0, 2].item()
    p.cache.table[0, 1, 0, 2] = p.cache.n_pages
    p.lm = p.lm.clone()
    p.lm[bad] = -math.inf
    check([0, 3, 6, 9, 12], [(0, 0, 3), (1, 3, 6), (2, 6, 9), (3, 9, 12)])
    # a length past the table is cut there
    p.cache.lens[0, 3, 1] = 32 * p.cache.max_pages + 5
    f(0, q.cuda(), cu_prefix=torch.tensor([0, 3, 6, 9, 12], dtype=torch.int32, device="cuda"))
    with pytest.raises(gk.GraceKVError):
        f.status()


@pytest.mark.parametrize("dtype,quant", KINDS)
def test_repeats_streams_and_graphs(gk, dtype, quant):
    f, q, out, cu = attend(gk, [[[30, 40]] * 40], [[[3000, 900], [20, 5000]]], cu=[0, 25, 40], dtype=dtype, quant=(quant, quant), seed=15)
    qd = q.cuda()
    for _ in range(3):
        assert torch.equal(f(0, qd, cu_prefix=cu), out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = f(0, qd, cu_prefix=cu, stream=s)
    s.synchronize()
    assert torch.equal(got, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        og = f(0, qd, cu_prefix=cu)
    f.prefix.lens[0, 0, 0] = 9                 # a replay goes by the lengths and groups that are there
    cu.copy_(torch.tensor([0, 2, 30], dtype=torch.int32))
    g.replay()
    new = f(0, qd, cu_prefix=cu)
    assert torch.equal(og, new) and not torch.equal(og, out)
    f.status()
    # outputs where the caller wants them
    mine = torch.empty_like(out)
    assert f(0, qd, cu_prefix=cu, out=mine) is mine and torch.equal(mine, new)


def test_no_requests_of_a_slot_and_no_entries(gk):
    attend(gk, np.zeros((1, 5, 2), int), np.zeros((1, 1, 2), int), seed=16)
    attend(gk, np.full((1, 5, 2), 9), [[[50, 60]]], cu=[2, 2], seed=17)


def test_a_prefix_in_the_requests_own_pool(gk):
    # one pool of pages, two tables: a request and the prefix that it was compressed to
    K, V = (torch.randn(40, 16, 64, device="cuda").to(BF) for _ in range(2))
    order = torch.randperm(40, device="cuda").to(torch.int32)
    own = gk.PagedCache(K, V, order[:12].view(1, 3, 2, 2), torch.tensor([[[20, 5], [0, 32], [17, 1]]], dtype=torch.int32, device="cuda"), Hq=4)
    pre = gk.PagedCache(K, V, order[12:36].view(1, 1, 2, 12), torch.tensor([[[190, 77]]], dtype=torch.int32, device="cuda"), Hq=4)
    q = queries(3, 4, 64, BF, 18)
    f = gk.SharedAttention(own, pre)
    out = f(0, q.cuda())
    f.status()

    class S:
        def __init__(s, c):
            s.c, s.lens = c, c.lens.cpu().numpy()

        def rows(s, i):
            n, t = int(s.lens[i]), s.c.table.cpu()[i]
            return R.entries(K.cpu(), t, n).double(), R.entries(V.cpu(), t, n).double(), torch.zeros(n).double()
    want, tol = expected(q, S(own), S(pre), [0, 3])
    assert ((out.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [5, 40])
def test_long_runs_of_tiles(gk, quant, d, B):
    """Pieces of fifty key tiles and more, read from memory rather than L2: rings turn many times, tiles land out of order.

    The values are independent of the weights, so an output is a sum of terms w v of random signs, and rounding every
    w by at most 2^-8 of itself moves it by a sum of such terms 2^-8 as large: 2^-8 of the outputs in norm, and as much
    again for rounding them."""
    G, gq, n, ps = 8, 4, 131072, 64
    g = torch.Generator(device="cuda").manual_seed(B)
    pool = []
    for _ in range(2):
        x = torch.empty(G * n // ps, ps, d, dtype=BF, device="cuda").normal_(generator=g)
        pool.append(x)
    real_kv = [x.float() for x in pool]
    sc = {}
    if quant:
        for i, name in enumerate(("k_scale", "v_scale")):
            e = torch.randint(117, 121, pool[i].shape[:2], generator=g, device="cuda", dtype=torch.int32)
            s = (e << 23).view(torch.float32).unsqueeze(-1)
            pool[i] = (real_kv[i] / s).clamp(-448, 448).to(torch.float8_e4m3fn)
            real_kv[i] = pool[i].float() * s
            sc[name] = e.to(torch.uint8)
        sc["dtype"] = BF
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.randperm(G * n // ps, generator=g, device="cuda").to(torch.int32).view(1, 1, G, -1)
    prefix = gk.PagedCache(*pool, table, torch.full((1, 1, G), n - 37, **i32), Hq=G * gq, **sc)
    own = gk.PagedCache(torch.zeros(1, 16, d, dtype=BF, device="cuda"), torch.zeros(1, 16, d, dtype=BF, device="cuda"),
                        torch.full((1, B, G, 1), -1, **i32), torch.zeros(1, B, G, **i32), Hq=G * gq)
    q = torch.empty(B, G * gq, d, dtype=BF, device="cuda").normal_(generator=g)
    f = gk.SharedAttention(own, prefix)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(3):
        flush.zero_()
        outs.append(f(0, q))
    f.status()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    for h in range(G):
        k, v = (x[table[0, 0, h].long()].view(n, d)[:n - 37].double() for x in real_kv)
        x = q[:, h * gq:(h + 1) * gq].reshape(-1, d).double() @ k.T / math.sqrt(d)
        want = (torch.softmax(x, dim=1) @ v).view(B, gq, d)
        got = outs[0][:, h * gq:(h + 1) * gq].double()
        assert float((got - want).norm() / want.norm()) < 2.0 ** -7
