"""Quantised pages: load, append, and the calls that read entries back
(gracekv_quant_load / _append, gracekv_paged_read / _unload) against their
definitions in 64 bits.  Without a rotation the codes are those of the
definition; rotated keys are the rounding of something within the rotation's
own error."""
import math

import numpy as np
import pytest
import torch

from . import quant_reference as Q
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


def cache(gk, lens, ps, Hq, d, dtype, seed=0, quant=True, logm=True, base=0.0, extra=3):
    """A cache of scattered pages for lens [L, B, G]; its pools hold a mark everywhere."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    table, pages = R.scattered_table(rng, lens, ps, extra)
    shape = (pages, ps, d)
    if quant:
        K, V = (torch.full(shape, m, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for m in (0x5a, 0xa5))
        sc = dict(k_scale=torch.full(shape[:2], 99, dtype=torch.uint8, device="cuda"),
                  v_scale=torch.full(shape[:2], 98, dtype=torch.uint8, device="cuda"), dtype=dtype)
    else:
        K, V = (torch.full(shape, m, dtype=dtype, device="cuda") for m in (7.0, -7.0))
        sc = {}
    return gk.PagedCache(K, V, table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), Hq=Hq, rope_base=base,
                         log_m=torch.full(shape[:2], 5.0, device="cuda") if logm else None, **sc)


def held(c):
    """Which pool rows the sequences hold."""
    table, lens = c.table.cpu(), c.lens.cpu()
    h = torch.zeros(c.n_pages * c.page_size, dtype=torch.bool)
    for i in np.ndindex(*lens.shape):
        e = torch.arange(int(lens[i]))
        h[table[i][e // c.page_size].long() * c.page_size + e % c.page_size] = True
    return h


def stored(c, name, i):
    """What sequence i's rows of K or V stand for, and their e."""
    n = int(c.lens[i])
    row = c.table[i].cpu()
    pool, scale = getattr(c, name).cpu(), getattr(c, name.lower() + "_scale").cpu()
    codes = R.entries(pool.view(torch.uint8), row, n).view(torch.float8_e4m3fn)
    sc = R.entries(scale, row, n)
    return Q.values(codes, sc), sc.numpy().astype(int) - 127


def rows(seed, n, d, dtype):
    """Rows of sizes from 2^-20 to 2^20, some with zeros, all of one sign, or one large value."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d, generator=g) * torch.exp2(40 * torch.rand(n, 1, generator=g) - 20)
    x[::7] = 0
    x[1::5, 3] *= 1000
    x[2::5, ::2] = 0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L,B,G,ps", [(1, 1, 1, 16), (2, 3, 2, 32), (5, 2, 3, 48), (3, 4, 8, 64)])
def test_load_and_unload(gk, dtype, d, L, B, G, ps):
    rng = np.random.default_rng(L * 100 + G)
    n = rng.integers(0, 90, (L, G))
    n[0, 0] = 0 if L > 1 else 33
    lens = np.zeros((L, B, G), int)
    lens[:, B - 1] = n
    c = cache(gk, lens, ps, G, d, dtype, seed=L)
    c.lens.zero_()
    off = np.concatenate([[0], np.cumsum(n)])
    E = int(off[-1])
    K, V, m = rows(1, E, d, dtype), rows(2, E, d, dtype), torch.rand(E)
    c.load_packed(B - 1, K.cuda(), V.cuda(), m.cuda(), torch.from_numpy(off).cuda())
    c.status()
    assert np.array_equal(c.lens.cpu().numpy(), lens)
    for l, g in np.ndindex(L, G):
        a, z = off[l * G + g], off[l * G + g + 1]
        for name, x in (("K", K), ("V", V)):
            got, e = stored(c, name, (l, B - 1, g))
            want, we = Q.quantised(x[a:z].double().numpy())
            assert np.array_equal(got, want) and np.array_equal(e, we[:, 0])
        assert torch.equal(R.entries(c.log_m.cpu(), c.table[l, B - 1, g].cpu(), z - a), m[a:z])
    h = held(c)
    for t, mark in ((c.K, 0x5a), (c.V, 0xa5), (c.k_scale, 99), (c.v_scale, 98)):
        assert (t.cpu().view(torch.uint8).view(h.numel(), -1)[~h] == mark).all()
    # back: the values themselves, exact in the rows' type
    back = c.unload_packed(B - 1, E)
    c.status()
    assert np.array_equal(back[0].double().cpu().numpy(), Q.quantised(K.double().numpy())[0])
    assert np.array_equal(back[1].double().cpu().numpy(), Q.quantised(V.double().numpy())[0])
    assert torch.equal(back[2].cpu(), m) and np.array_equal(back[3].cpu().numpy(), off)
    # and written again they stay what they are
    c2 = cache(gk, lens, ps, G, d, dtype, seed=L + 50)
    c2.load_packed(B - 1, *back)
    again = c2.unload_packed(B - 1, E)
    assert all(torch.equal(x, y) for x, y in zip(back, again))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_at_the_borders(gk, dtype):
    d, big = 64, torch.finfo(dtype).max
    cases = [[0.0], [448.0], [449.0 if dtype == F32 else 450.0], [-448.0, 447.0], [2.0 ** -9], [2.0 ** -10], [3 * 2.0 ** -11], [big], [-big, 1.0],
             [448 * 2.0 ** 119], [2.0 ** -126], [448 * 2.0 ** -120, 2.0 ** -126], [2.0 ** -130], [math.inf, 1.0], [-math.inf], [math.nan],
             [math.nan, math.inf, 3.0, -5.0], [240.0, 248.0, 232.0, 17.0, 19.0, 1.0625, 1.1875], [2.0 ** 40, 2.0 ** 33, 2.0 ** 31]]
    x = torch.zeros(len(cases), d)
    for i, v in enumerate(cases):
        x[i, 5:5 + len(v)] = torch.tensor(v)
    x = x.to(dtype)
    n = len(cases)
    c = cache(gk, [[[n]]], 16, 1, d, dtype, logm=False)
    c.load_packed(0, x.cuda(), x.flip(1).contiguous().cuda(), None, torch.tensor([0, n], device="cuda"))
    back = c.unload_packed(0, n)
    c.status()
    want, e = Q.quantised(x.double().numpy())
    assert np.array_equal(stored(c, "K", (0, 0, 0))[1], e[:, 0])
    assert np.array_equal(back[0].double().cpu().numpy(), want, equal_nan=True)
    assert np.array_equal(back[1].double().cpu().numpy(), want[:, ::-1], equal_nan=True)
    assert (back[2] == 0).all()


def fused(N, G, Hq, d, dtype, seed):
    """q, k, v as slices of one projection's rows."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, (Hq + 2 * G) * d, generator=g).to(dtype).cuda()
    q, k, v = x.split([Hq * d, G * d, G * d], dim=1)
    return q.view(N, Hq, d), k.view(N, G, d), v.view(N, G, d)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,G,Hq,ps,base", [((1,), 1, 1, 16, 1e4), ((1, 0, 5), 2, 8, 32, 5e5), ((40, 3, 0, 130), 3, 9, 48, 1e4),
                                             ((3000, 411), 8, 32, 64, 5e5), ((7, 9), 2, 14, 16, 0.0)])
def test_append_and_read(gk, dtype, d, new, G, Hq, ps, base):
    rng = np.random.default_rng(len(new) + d)
    B, N = len(new), sum(new)
    before = rng.integers(0, 50, (2, B, G))
    lens = before + np.array(new)[None, :, None]
    c = cache(gk, lens, ps, Hq, d, dtype, seed=d, base=base)
    q, k, v = fused(N, G, Hq, d, dtype, 3)
    pos = torch.from_numpy(rng.integers(0, 200000, N).astype(np.int32))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I32)
    out = c.append(1, k, v, pos.cuda(), q=q, cu_new=cu)
    kk, vv = c.read(1, N, cu=cu)
    c.status()
    want = R.rotate(q, pos, base)
    assert ((out.double().cpu() - want).abs() <= R.rotate_bound(q, want, R.BITS_BF16 if dtype == BF else R.BITS_F32)).all()
    rk, slack = R.rotate(k, pos, base).numpy(), 0.0
    if base:
        slack = R.rotate_bound(k, torch.zeros(()), 8).numpy()
    t = 0
    written = held(c)
    for b, n in enumerate(new):
        for g in range(G):
            got, e = stored(c, "K", (1, b, g))
            x, s = rk[t:t + n, g], slack[t:t + n, g] if base else 0.0
            assert Q.between(got[lens[1, b, g] - n:], x, s, e[lens[1, b, g] - n:]).all()
            top = np.abs(x).max(-1) if n else np.zeros(0)
            ts = np.max(s, -1) if base else 0.0
            assert ((e[lens[1, b, g] - n:] >= Q.exponent(top - ts)) & (e[lens[1, b, g] - n:] <= Q.exponent(top + ts))).all()
            assert np.array_equal(kk[t:t + n, g].double().cpu().numpy(), got[lens[1, b, g] - n:])
            got, e = stored(c, "V", (1, b, g))
            assert np.array_equal(got[lens[1, b, g] - n:], Q.quantised(v[t:t + n, g].double().cpu().numpy())[0])
            assert np.array_equal(vv[t:t + n, g].double().cpu().numpy(), got[lens[1, b, g] - n:])
            assert (R.entries(c.log_m.cpu(), c.table[1, b, g].cpu(), int(lens[1, b, g]))[int(before[1, b, g]):] == 0).all()
        t += n
    # nothing else was written: the entries before, the other layer, other pages
    for b, g in np.ndindex(B, G):
        e = torch.arange(int(before[1, b, g]), int(lens[1, b, g]))
        written[c.table[1, b, g].cpu()[e // ps].long() * ps + e % ps] = False
        e = torch.arange(int(before[1, b, g]))
        assert (R.entries(c.k_scale.cpu(), c.table[1, b, g].cpu(), int(before[1, b, g])) == 99).all()
    assert (c.k_scale.cpu().view(-1)[written] == 99).all() and (c.K.cpu().view(torch.uint8).view(-1, d)[written] == 0x5a).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("quant", [True, False])
def test_read_sides(gk, dtype, quant):
    # whole sequences by their lengths, more rows than entries, one row of each, no rows, given tensors of other strides
    lens = np.array([[[5, 5], [0, 0], [17, 17]], [[3, 8], [1, 0], [40, 2]]])
    c = cache(gk, lens, 16, 4, 64, dtype, quant=quant)
    g = torch.Generator().manual_seed(0)
    data = {}
    for i in np.ndindex(*lens.shape):
        n = int(lens[i])
        x = torch.randn(2, n, 64, generator=g).to(dtype)
        data[i] = Q.quantised(x.double().numpy())[0] if quant else x.double().numpy()
        e = torch.arange(n)
        at = c.table[i].cpu()[e // 16].long() * 16 + e % 16
        for name, y in zip("KV", x):
            if quant:
                codes, sc = Q.pool(y)
                getattr(c, name).view(torch.uint8).view(-1, 64)[at.cuda()] = codes.view(torch.uint8).cuda()
                getattr(c, name.lower() + "_scale").view(-1)[at.cuda()] = sc.cuda()
            else:
                getattr(c, name).view(-1, 64)[at.cuda()] = y.cuda()
    for l, counts in ((0, (5, 0, 17)), (1, (4, 2, 40)), (1, (0, 0, 0)), (0, (1, 0, 0))):
        N = sum(counts) + 2
        cu = torch.tensor(np.concatenate([[1], 1 + np.cumsum(counts)]), **I32)       # a row of no request at each end
        wide = torch.full((2, N, 2, 3 * 64), 9.0, dtype=dtype, device="cuda")
        k, v = wide[0, :, :, 64:128], wide[1, :, :, :64]
        rk, rv = c.read(l, N, cu=cu, k=k, v=v)
        c.status()
        assert rk.data_ptr() == k.data_ptr() and rv.data_ptr() == v.data_ptr()
        want = np.full((2, N, 2, 3 * 64), 9.0)
        for b, n in enumerate(counts):
            for h in range(2):
                x = data[l, b, h][:, max(0, lens[l, b, h] - n):]
                x = np.concatenate([np.zeros((2, n - x.shape[1], 64)), x], axis=1)
                a = 1 + sum(counts[:b])
                want[0, a:a + n, h, 64:128], want[1, a:a + n, h, :64] = x
        assert np.array_equal(wide.double().cpu().numpy(), want)
    k, v = c.read(1, 3)                       # the last entry of every head
    for b, h in np.ndindex(3, 2):
        x = data[1, b, h][:, -1] if lens[1, b, h] else np.zeros((2, 64))
        assert np.array_equal(k[b, h].double().cpu().numpy(), x[0]) and np.array_equal(v[b, h].double().cpu().numpy(), x[1])
    assert c.read(0, 0, cu=torch.zeros(4, **I32))[0].shape == (0, 2, 64)
    # all of a request as a packed cache, room for more or for less
    for b in range(3):
        off = np.concatenate([[0], np.cumsum(lens[:, b].reshape(-1))])
        flat = np.concatenate([data[l, b, h] for l, h in np.ndindex(2, 2)], axis=1)
        for room in (int(off[-1]), int(off[-1]) + 5):
            out = tuple(torch.full(s, 9, dtype=t, device="cuda") for s, t in (((room, 64), dtype), ((room, 64), dtype), ((room,), F32),
                                                                             ((5,), torch.int64)))
            c.unload_packed(b, room, out)
            c.status()
            assert np.array_equal(out[3].cpu().numpy(), off)
            for x, y in zip(out[:2], flat):
                assert np.array_equal(x[:off[-1]].double().cpu().numpy(), y) and (x[off[-1]:] == 9).all()
            assert (out[2][:off[-1]] == 5).all() and (out[2][off[-1]:] == 9).all()


def test_read_back_into_the_prompts_attention(gk):
    # a chunk over a quantised cache: append, read the whole sequences, attend
    B, G, Hq, d, ps = 3, 2, 4, 64, 16
    old, new = np.array([33, 0, 70]), np.array([5, 9, 1])
    lens = np.broadcast_to((old + new)[None, :, None], (1, B, G))
    c = cache(gk, lens, ps, Hq, d, BF, base=1e4, logm=False)
    total = int((old + new).sum())
    cu_all = torch.tensor(np.concatenate([[0], np.cumsum(old + new)]), **I32)
    cu_new = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I32)
    q, k, v = fused(total, G, Hq, d, BF, 8)
    pos = torch.cat([torch.arange(n, **I32) for n in old + new])
    qr = c.append(0, k, v, pos, q=q, cu_new=cu_all)
    kk, vv = c.read(0, total, cu=cu_all)
    fresh = torch.cat([torch.arange(int(o), int(o + n)) + int(a) for o, n, a in zip(old, new, cu_all.cpu())]).cuda()
    qn = qr[fresh].contiguous()
    out = gk.PromptAttention(G=G, Hq=Hq, d=d, dtype=BF)(qn, kk, vv, cu_new, cu_all)
    want, _, tol, _ = R.prompt(qn, kk, vv, cu_new.tolist(), cu_all.tolist(), bf16=True)
    assert ((out.double().cpu() - want).abs() <= tol).all()


def test_words_that_do_not_fit(gk):
    lens = np.array([[[20, 20], [9, 9]]])
    c = cache(gk, lens, 16, 2, 64, BF)
    x, m = torch.randn(40, 64).to(BF).cuda(), torch.zeros(40, device="cuda")

    def reported():
        with pytest.raises(gk.GraceKVError) as e:
            c.status()
        assert e.value.status == gk.GKV_EINVAL
        c.status()

    # a page outside the pool: its entries are skipped, and read as zeros
    good = c.table.clone()
    c.table[0, 0, 1, 0] = c.n_pages
    c.load_packed(0, x, x, m, torch.tensor([0, 20, 40], device="cuda"))
    reported()
    back = c.unload_packed(0, 40)
    reported()
    want = Q.quantised(x.double().cpu().numpy())[0]
    want[20:36] = 0
    assert np.array_equal(back[0].double().cpu().numpy(), want)
    k, v = c.read(0, 20, cu=torch.tensor([0, 20, 20], **I32))
    reported()
    assert np.array_equal(k[:, 1].double().cpu().numpy(), want[20:]) and np.array_equal(k[:, 0].double().cpu().numpy(), want[:20])
    c.table.copy_(good)
    # offsets that run backwards cost no other head its entries
    c.load_packed(1, x, x, m, torch.tensor([0, 9, 3], device="cuda"))
    reported()
    assert c.lens[0, 1].tolist() == [9, 0]
    assert np.array_equal(stored(c, "K", (0, 1, 0))[0], Q.quantised(x[:9].double().cpu().numpy())[0])
    # cu words
    c.read(0, 5, cu=torch.tensor([0, 6, 5], **I32))
    reported()
    c.append(0, x[:10].view(5, 2, 64), x[:10].view(5, 2, 64), torch.zeros(5, **I32), cu_new=torch.tensor([3, 1, 5], **I32))
    reported()
    # more entries than there is room for, lengths past the table or below 0
    out = tuple(torch.full(s, 9, dtype=t, device="cuda") for s, t in (((30, 64), BF), ((30, 64), BF), ((30,), F32), ((3,), torch.int64)))
    c.load_packed(0, x, x, m, torch.tensor([0, 20, 40], device="cuda"))
    c.status()
    c.unload_packed(0, 25, tuple(t[:25] if t.numel() > 3 else t for t in out))
    reported()
    assert out[3].tolist() == [0, 20, 40] and (out[0][25:] == 9).all()
    assert np.array_equal(out[0][:25].double().cpu().numpy(), Q.quantised(x[:25].double().cpu().numpy())[0])
    c.lens[0, 0, 0] = 16 * c.max_pages + 1
    c.lens[0, 0, 1] = -3
    c.unload_packed(0, 16 * c.max_pages)
    reported()


def test_pages_that_the_cache_hands_out(gk):
    # load, unload, release, load into a cache of another kind of pages; appended tokens in between
    L, B, G, d = 2, 3, 2, 64
    one = gk.PagedCache.allocate(L=L, B=B, G=G, Hq=4, d=d, dtype=BF, n_pages=60, max_pages=6, page_size=16, quantised=True, rope_base=1e4)
    two = gk.PagedCache.allocate(L=L, B=B, G=G, Hq=4, d=d, dtype=BF, n_pages=60, max_pages=6, page_size=16)
    assert one.quantised and not two.quantised and one.dtype is BF
    n = np.array([3, 40, 0, 17])
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).cuda()
    K, V = rows(4, 60, d, BF).cuda(), rows(5, 60, d, BF).cuda()
    one.load(1, gk.Cache(K, V, None, torch.rand(60, device="cuda"), None, None, off), 60)
    one.advance()
    for l in range(L):
        one.append(l, torch.randn(B, G, d, device="cuda").to(BF), torch.randn(B, G, d, device="cuda").to(BF), torch.full((B,), 70, **I32))
    one.status()
    back = one.unload(1)
    one.status()
    assert back.K.shape == (64, d) and back.offsets.tolist() == [0, 4, 45, 46, 64]
    assert np.array_equal(back.K[:3].double().cpu().numpy(), Q.quantised(K[:3].double().cpu().numpy())[0])
    one.release(1)
    two.load(0, back, 64)
    again = two.unload(0)
    assert torch.equal(again.K, back.K) and torch.equal(again.V, back.V) and torch.equal(again.log_m, back.log_m)
    one.load(2, again, 64)
    third = one.unload(2)
    assert torch.equal(third.K, back.K) and torch.equal(third.log_m, back.log_m)
    with pytest.raises(gk.GraceKVError):
        one.unload(3)


def test_other_streams_and_graphs(gk):
    lens = np.array([[[30, 30], [7, 7]]])
    c = cache(gk, lens, 16, 4, 128, BF, base=1e4)
    q, k, v = fused(12, 2, 4, 128, BF, 1)
    cu, pos = torch.tensor([0, 9, 12], **I32), torch.arange(12, **I32)
    want = [t.clone() for t in (c.append(0, k, v, pos, q=q, cu_new=cu), *c.read(0, 12, cu=cu))]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    qs = c.append(0, k, v, pos, q=q, cu_new=cu, stream=s)
    ks, vs = c.read(0, 12, cu=cu, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (qs, ks, vs)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        qg = c.append(0, k, v, pos, q=q, cu_new=cu)
        kg, vg = c.read(0, 12, cu=cu)
    k.mul_(2)                                 # a replay reads what is there now; powers of two change the scale alone
    g.replay()
    c.status()
    assert torch.equal(qg, want[0]) and torch.equal(kg, want[1] * 2) and torch.equal(vg, want[2])
