"""The paged cache: load, advance, append and attention (gracekv_paged_*)
against their definitions in 64 bits (serving_reference, which also derives
the tolerances)."""
import math

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


def pool(seed, pages, ps, d, dtype, junk=None):
    g = torch.Generator().manual_seed(seed)
    K, V = (torch.randn(pages, ps, d, generator=g).to(dtype) for _ in range(2))
    lm = torch.log(torch.clamp(torch.exp2(1 + 6 * torch.rand(pages, ps, generator=g)) * torch.rand(pages, ps, generator=g), min=1.0))
    return K, V, lm


def spoil(t, table, lens):
    """Non-finite values in every pool row that no sequence holds."""
    ps = t.shape[1]
    held = torch.zeros(t.shape[0] * ps, dtype=torch.bool)
    for i in np.ndindex(*lens.shape):
        n = int(lens[i])
        e = torch.arange(n)
        held[table[i][e // ps].long() * ps + e % ps] = True
    flat = t.view(t.shape[0] * ps, -1)
    flat[~held] = math.nan
    odd = (~held).nonzero()[::2, 0]
    flat[odd] = math.inf
    return t


# ------------------------------------------------------------------ attention
def attend(gk, lens, ps, Hq, d, dtype, seed=0, logm=True, l=0, edit=None, q_scale=1.0):
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    table, pages = R.scattered_table(rng, lens, ps)
    K, V, lm = pool(seed, pages, ps, d, dtype)
    if edit:
        edit(K, V, lm, table)
    for t in (K, V, lm):
        spoil(t, table, lens)
    lens_t = torch.from_numpy(lens.astype(np.int32))
    g = torch.Generator().manual_seed(seed + 1)
    q = torch.randn(lens.shape[1], Hq, d, generator=g)
    q[:, 1::2] *= 3
    q = (q * q_scale).to(dtype)
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), lens_t.cuda(), log_m=lm.cuda() if logm else None, Hq=Hq)
    out = c.attention(l, q.cuda())
    c.status()
    want, tol = R.decode(q, K, V, lm if logm else None, table, lens_t, l, bf16=dtype == BF)
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    err = (got - want).abs()
    assert (err <= tol).all(), f"{float((err - tol).max()):.3e} over its bound"
    assert (got[want == 0] == 0).all()
    return c, q, out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1025])
def test_attention_lengths(gk, dtype, d, n):
    attend(gk, [[[n, max(0, n - 1)]]], 64, 8, d, dtype, seed=n)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps", [16, 32, 48, 64, 80, 128, 256])
def test_attention_page_sizes(gk, dtype, ps):
    attend(gk, [[[77, 0], [300, 5], [ps, 2 * ps], [ps - 1, ps + 1]]], ps, 4, 128, dtype, seed=ps)
    attend(gk, [[[77, 0], [300, 5], [ps, 2 * ps], [ps - 1, ps + 1]]], ps, 4, 64, dtype, seed=ps, logm=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,G", [(1, 1), (6, 3), (6, 2), (4, 1), (10, 2), (6, 1), (14, 2), (8, 1), (32, 8)])
def test_attention_head_layouts(gk, dtype, Hq, G):
    lens = np.random.default_rng(G).integers(0, 400, (1, 3, G))
    attend(gk, lens, 32, Hq, 128, dtype, seed=Hq)
    attend(gk, lens, 32, Hq, 64, dtype, seed=Hq)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_uneven_and_long(gk, dtype):
    # one sequence far longer than the others: split over many CTAs and joined
    attend(gk, [[[40000, 3], [0, 900], [1, 7000]]], 64, 8, 128, dtype, seed=2)
    attend(gk, [[[40000, 3], [0, 900], [1, 7000]]], 16, 8, 64, dtype, seed=3)


def test_attention_many_sequences(gk):
    lens = np.random.default_rng(5).integers(0, 130, (1, 300, 8))
    attend(gk, lens, 32, 32, 64, BF, seed=5)
    attend(gk, np.zeros((1, 40, 4), int), 32, 4, 64, BF, seed=6)


def test_attention_reads_its_layer(gk):
    lens = np.random.default_rng(7).integers(0, 200, (3, 2, 2))
    for l in range(3):
        attend(gk, lens, 16, 4, 64, BF, seed=7, l=l)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_log_m_extremes(gk, dtype):
    low = torch.finfo(torch.float32).min

    def some(K, V, lm, table):
        lm[:, ::3] = -math.inf           # multiplicity 0: not seen
        lm[:, 1::3] = low                # the type's lowest value: no weight beside the others

    attend(gk, [[[90, 200], [1000, 17]]], 16, 8, 128, dtype, seed=8, edit=some)

    def none(K, V, lm, table):
        lm.fill_(-math.inf)

    c, q, out = attend(gk, [[[90, 200], [1000, 17]]], 16, 8, 128, dtype, seed=9, edit=none)
    assert (out == 0).all()

    def lowest(K, V, lm, table):          # equal logits of the lowest value: the mean
        lm.fill_(low)

    attend(gk, [[[90, 200], [1000, 17]]], 16, 8, 128, dtype, seed=10, edit=lowest)

    def big(K, V, lm, table):
        lm.mul_(40.0)

    attend(gk, [[[90, 200], [1000, 17]]], 16, 8, 128, dtype, seed=11, edit=big)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_large_logits(gk, dtype):
    attend(gk, [[[900, 33]]], 64, 8, 128, dtype, seed=12, q_scale=30.0)


def test_attention_is_the_same_every_time(gk):
    for dtype in (BF, F32):
        c, q, out = attend(gk, [[[5000, 3], [200, 900], [1, 7000]]], 64, 8, 128, dtype, seed=13)
        q = q.cuda()
        for _ in range(5):
            assert torch.equal(c.attention(0, q), out)


def test_attention_offsets_past_32_bits(gk):
    # the last pages of a pool of more than 2^32 bytes and 2^31 elements
    ps, d = 128, 128
    pages = (1 << 31) // (ps * d) + 40
    K = torch.empty(pages, ps, d, dtype=BF, device="cuda")
    V = torch.empty(pages, ps, d, dtype=BF, device="cuda")
    n = 1000
    held = torch.arange(pages - 8, pages, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in (K, V):
        t[held] = torch.empty(8, ps, d, dtype=BF, device="cuda").normal_(generator=g)
    table = held.flip(0).to(torch.int32).view(1, 1, 1, 8).contiguous()
    lens = torch.tensor([[[n]]], **I32)
    c = gk.PagedCache(K, V, table, lens, Hq=4)
    q = torch.empty(1, 4, d, dtype=BF, device="cuda").normal_(generator=g)
    out = c.attention(0, q)
    c.status()
    small = torch.arange(8, dtype=torch.int32).view(1, 1, 1, 8)
    want, tol = R.decode(q, K[held.flip(0)], V[held.flip(0)], None, small, lens, 0, bf16=True)
    assert ((out.double().cpu() - want).abs() <= tol).all()
    # append there too: the row after the last
    c.advance_by(torch.tensor([0, 1], **I32))
    new = torch.empty(1, 1, d, dtype=BF, device="cuda").normal_(generator=g)
    c.append(0, new, new, torch.zeros(1, **I32))
    c.status()
    page, row = int(table[0, 0, 0, n // ps]), n % ps
    assert torch.equal(K[page, row], new[0, 0]) and torch.equal(V[page, row], new[0, 0])


def test_attention_reports_pages_outside_the_pool(gk):
    for dtype in (BF, F32):
        K, V, lm = (t.cuda() for t in pool(1, 6, 32, 64, dtype))
        q = torch.randn(2, 4, 64).to(dtype).cuda()
        for table, lens in [([[0, 1, 6], [3, 4, 5]], [96, 96]), ([[0, -1, 2], [3, 4, 5]], [70, 96]),
                            ([[0, 1, 2], [3, 4, 5]], [97, 96]), ([[0, 1, 2], [3, 4, 5]], [1 << 30, 5])]:
            c = gk.PagedCache(K, V, torch.tensor(table, **I32).view(1, 2, 1, 3), torch.tensor(lens, **I32).view(1, 2, 1),
                              log_m=lm, Hq=4)
            out = c.attention(0, q)
            with pytest.raises(gk.GraceKVError) as e:
                c.status()
            assert e.value.status == gk.GKV_EINVAL
            c.status()
            # the other request is as it should be
            want, tol = R.decode(q, K, V, lm, c.table, c.lens.clamp(max=96), 0, bf16=dtype == BF) if table[0] == [0, 1, 2] else (None, None)
            if want is not None:
                assert ((out.double().cpu() - want).abs() <= tol)[1].all()
        # a negative length is an idle slot
        c = gk.PagedCache(K, V, torch.zeros(1, 2, 1, 3, **I32), torch.tensor([[[-5], [3]]], **I32), Hq=4)
        assert (c.attention(0, q)[0] == 0).all()


def test_attention_on_another_stream_and_in_a_graph(gk):
    c, q, out = attend(gk, [[[700, 3], [200, 900]]], 64, 8, 128, BF, seed=14)
    q = q.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    there = c.attention(0, q, stream=s)
    c.status(s)
    assert torch.equal(there, out)
    buf = torch.empty_like(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attention(0, q, out=buf)
    buf.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(buf, out)


# --------------------------------------------------------------------- append
def append_case(gk, counts, before, ps, Hq, G, d, dtype, base, pos, seed=0, with_q=True, strided=False, l=1):
    rng = np.random.default_rng(seed)
    counts, before = np.asarray(counts), np.asarray(before)
    B = len(counts)
    lens = np.zeros((2, B, G), np.int64)
    lens[l] = before + counts[:, None]
    table, pages = R.scattered_table(rng, lens, ps)
    K, V, lm = pool(seed, pages, ps, d, dtype)
    N = int(counts.sum())
    g = torch.Generator().manual_seed(seed + 1)
    q, k, v = (torch.randn(N, h, d, generator=g).to(dtype) for h in (Hq, G, G))
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    if strided:
        f = torch.cat([t.reshape(N, -1) for t in (q, k, v)], 1).cuda()
        qd, kd, vd = (t.view(N, -1, d) for t in f.split([Hq * d, G * d, G * d], 1))
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), log_m=lm.cuda(),
                      Hq=Hq, rope_base=base)
    pos = torch.as_tensor(pos, dtype=torch.int32)
    qr = c.append(l, kd, vd, pos.cuda(), q=qd if with_q else None, cu_new=cu)
    c.status()
    bits = R.BITS_BF16 if dtype == BF else R.BITS_F32
    if with_q:
        want = R.rotate(q, pos, base)
        assert ((qr.double().cpu() - want).abs() <= R.rotate_bound(q, want, bits)).all()
    want = R.rotate(k, pos, base)
    tol = R.rotate_bound(k, want, bits)
    wK, wT, wV, wm = K.double(), torch.zeros_like(K, dtype=torch.float64), V.clone(), lm.clone()
    t = 0
    for b in range(B):
        for j in range(counts[b]):
            for h in range(G):
                idx = int(lens[l, b, h] - counts[b] + j)
                if idx < 0:
                    continue
                page = int(table[l, b, h, idx // ps])
                wK[page, idx % ps], wT[page, idx % ps] = want[t, h], tol[t, h]
                wV[page, idx % ps], wm[page, idx % ps] = v[t, h], 0.0
            t += 1
    assert ((c.K.double().cpu() - wK).abs() <= wT).all()       # everything else bit for bit
    assert torch.equal(c.V.cpu(), wV) and torch.equal(c.log_m.cpu(), wm)
    return c


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("base", [1e4, 5e5, 0.0])
def test_append(gk, dtype, d, base):
    counts = [1, 0, 17, 130, 1]
    before = [[5, 0], [9, 2], [0, 31], [100, 63], [15, 16]]
    pos = np.random.default_rng(1).integers(0, 131072, 149)
    append_case(gk, counts, before, 16, 8, 2, d, dtype, base, pos, strided=True)
    append_case(gk, counts, before, 64, 4, 2, d, dtype, base, pos, with_q=False)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,G", [(1, 1), (6, 3), (14, 2), (8, 1), (5, 5)])
def test_append_head_layouts(gk, dtype, Hq, G):
    append_case(gk, [3, 1], np.full((2, G), 7), 10, Hq, G, 64, dtype, 1e4, [0, 1, 2, 9])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_positions(gk, dtype):
    # large, negative and extreme positions keep the angle
    pos = [0, 1, -1, 3, 131071, 1 << 20, (1 << 24) + 1, (1 << 31) - 1, -(1 << 31), 77777777]
    append_case(gk, [10], [[4]], 32, 2, 1, 128, dtype, 5e5, pos)
    append_case(gk, [10], [[4]], 32, 2, 1, 64, dtype, 1e4, pos)
    append_case(gk, [10], [[4]], 32, 2, 1, 64, dtype, 1.0, pos)


def test_append_a_long_prompt(gk):
    append_case(gk, [3000, 1], [[0, 40], [2, 2]], 48, 4, 2, 128, BF, 5e5, np.arange(3001))


def test_append_of_single_tokens(gk):
    # no cu_new: token b is request b's; idle requests (length 0) store nothing
    K, V, lm = pool(2, 8, 16, 64, BF)
    lens = torch.tensor([[[17, 3], [0, 0], [1, 16]]], dtype=torch.int32)
    table, pages = R.scattered_table(np.random.default_rng(3), lens.numpy(), 16)
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), lens.cuda(), log_m=lm.cuda(), Hq=4)
    k, v = (torch.randn(3, 2, 64).to(BF) for _ in range(2))
    c.append(0, k.cuda(), v.cuda(), torch.zeros(3, **I32))
    c.status()
    for b in range(3):
        for g in range(2):
            n = int(lens[0, b, g])
            if n:
                page, row = int(table[0, b, g, (n - 1) // 16]), (n - 1) % 16
                K[page, row], V[page, row], lm[page, row] = k[b, g], v[b, g], 0.0
    assert torch.equal(c.K.cpu(), K) and torch.equal(c.V.cpu(), V) and torch.equal(c.log_m.cpu(), lm)


def test_append_into_a_dense_cache(gk):
    # pages of T entries: the [L, G, T, d] keys and values that the compressor takes
    L, G, T, d, Hq = 2, 2, 100, 64, 4
    K, V = (torch.zeros(L, G, T, d, dtype=BF, device="cuda") for _ in range(2))
    table = torch.arange(L * G, **I32).view(L, 1, G, 1)
    c = gk.PagedCache(K.view(L * G, T, d), V.view(L * G, T, d), table, torch.full((L, 1, G), T, **I32), Hq=Hq, rope_base=1e4)
    cu, pos = torch.tensor([0, T], **I32), torch.arange(T, **I32)
    for l in range(L):
        k, v, q = (torch.randn(T, h, d).to(BF) for h in (G, G, Hq))
        qr = c.append(l, k.cuda(), v.cuda(), pos, q=q.cuda(), cu_new=cu, out=None)
        want = R.rotate(k, pos, 1e4)
        assert ((K[l].transpose(0, 1).double().cpu() - want).abs() <= R.rotate_bound(k, want, R.BITS_BF16)).all()
        assert torch.equal(V[l].transpose(0, 1).cpu(), v)
        qin = q.cuda()
        assert c.append(l, k.cuda(), v.cuda(), pos, q=qin, cu_new=cu, out=qin) is qin      # in place
        assert torch.equal(qin, qr)
    c.status()


def test_append_reports_what_it_does_not_follow(gk):
    K, V, _ = pool(4, 4, 16, 64, BF)
    k, v = (torch.randn(2, 1, 64).to(BF) for _ in range(2))
    for table, lens in [([4, 1], [3, 3]), ([-1, 1], [3, 3]), ([0, 1], [40, 3])]:
        c = gk.PagedCache(K.cuda(), V.cuda(), torch.tensor(table, **I32).view(1, 2, 1, 1), torch.tensor(lens, **I32).view(1, 2, 1), Hq=1)
        c.append(0, k.cuda(), v.cuda(), torch.zeros(2, **I32))
        with pytest.raises(gk.GraceKVError) as e:
            c.status()
        assert e.value.status == gk.GKV_EINVAL
        want = K.clone()
        want[1, 2] = k[1, 0]
        assert torch.equal(c.K.cpu(), want)


def test_advance(gk):
    lens = torch.tensor([[[3, 0], [0, 0], [7, 9]], [[1, 1], [0, 0], [2, 0]]], dtype=torch.int32)
    K = torch.zeros(4, 16, 64, dtype=BF, device="cuda")
    c = gk.PagedCache(K, K.clone(), torch.zeros(2, 3, 2, 1, **I32), lens.cuda(), Hq=2)
    c.advance()
    assert torch.equal(c.lens.cpu(), lens + (lens > 0))
    cu = c.advance([2, 0, 5])
    assert cu.tolist() == [0, 2, 2, 7]
    assert torch.equal(c.lens.cpu(), lens + (lens > 0) + torch.tensor([2, 0, 5], dtype=torch.int32)[None, :, None])


# ----------------------------------------------------------------------- load
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ps", [16, 50, 64])
@pytest.mark.parametrize("logm", [True, False])
def test_load(gk, dtype, d, ps, logm):
    L, B, G, b = 3, 2, 2, 1
    rng = np.random.default_rng(ps)
    n = np.array([0, 1, ps, ps + 1, 333, 0])
    held = np.zeros((L, B, G), np.int64)
    held[:, b] = n.reshape(L, G)
    table, pages = R.scattered_table(rng, held, ps)
    K, V, lm = pool(ps, pages, ps, d, dtype)
    g = torch.Generator().manual_seed(1)
    E = int(n.sum())
    k, v = (torch.randn(E, d, generator=g).to(dtype) for _ in range(2))
    m = torch.rand(E, generator=g)
    off = np.concatenate([[0], np.cumsum(n)])
    c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.full((L, B, G), 9, **I32), log_m=lm.cuda(), Hq=G)
    c.load_packed(b, k.cuda(), v.cuda(), m.cuda() if logm else None, torch.from_numpy(off).cuda())
    c.status()
    for i in range(L * G):
        for j in range(n[i]):
            page, row = int(table[i // G, b, i % G, j // ps]), j % ps
            K[page, row], V[page, row], lm[page, row] = k[off[i] + j], v[off[i] + j], m[off[i] + j] if logm else 0.0
    assert torch.equal(c.K.cpu(), K) and torch.equal(c.V.cpu(), V) and torch.equal(c.log_m.cpu(), lm)
    held[:, 0] = 9
    assert np.array_equal(c.lens.cpu().numpy(), held)


def test_load_reports_what_does_not_fit(gk):
    ps, E = 16, 40
    K, V, lm = pool(1, 6, ps, 64, BF)
    k, v = (torch.randn(E, 64).to(BF) for _ in range(2))
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32).view(1, 1, 2, 2)
    for off, lens in [([0, 20, 41], [20, 0]), ([0, 20, 10], [20, 0]), ([-2, 20, 40], [0, 20]), ([0, 0, 40], [0, 32])]:
        c = gk.PagedCache(K.cuda(), V.cuda(), table.cuda(), torch.zeros(1, 1, 2, **I32), log_m=lm.cuda(), Hq=2)
        c.load_packed(0, k.cuda(), v.cuda(), None, torch.tensor(off, device="cuda"))
        with pytest.raises(gk.GraceKVError) as e:
            c.status()
        assert e.value.status == gk.GKV_EINVAL
        assert c.lens.view(-1).tolist() == lens
        assert torch.equal(c.K[4:].cpu(), K[4:])


# ------------------------------------------------------------- pages, refusals
def test_pages_are_handed_out_and_come_back(gk):
    c = gk.PagedCache.allocate(L=2, B=3, G=2, Hq=4, d=64, dtype=BF, n_pages=40, max_pages=5, page_size=16, rope_base=1e4)
    rng = np.random.default_rng(0)

    def packed(n):
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
        E = int(off[-1])
        pk = gk.Cache.empty(E, 64, 4, BF)
        pk.K.normal_(), pk.V.normal_(), pk.log_m.zero_()
        pk.offsets.copy_(torch.from_numpy(off))
        return pk, E

    def consistent():
        lens, table = c.lens.cpu().numpy(), c.table.cpu().numpy()
        assert np.array_equal(lens, c._host_lens)
        used = [p for i in np.ndindex(*lens.shape) for p in table[i][:-(-lens[i] // 16)]]
        assert len(used) == len(set(used)) and all(0 <= p < 40 for p in used)
        return len(used)

    pk, E = packed([16, 17, 0, 3])
    c.load(1, pk, E)
    assert consistent() == 4
    c.load(2, *packed([33, 1, 1, 1]))
    for step in range(20):
        counts = None if step % 2 else rng.integers(0, 3, 3) * [0, 1, 1]
        cu = c.advance(counts)
        N = 3 if cu is None else int(cu[-1])
        for l in range(2):
            k = torch.randn(N, 2, 64).to(BF).cuda()
            c.append(l, k, k, torch.arange(N, **I32), cu_new=cu)
        consistent()
    c.status()
    # what request 1 was loaded with is still there
    got = R.entries(c.K.cpu(), c.table[0, 1, 1].cpu(), 17)
    assert torch.equal(got, pk.K[16:33].cpu())
    free = c._n_free
    with pytest.raises(gk.GraceKVError) as e:
        c.advance([1000, 0, 0])
    assert e.value.status == gk.GKV_ECAPACITY and c._n_free == free
    with pytest.raises(gk.GraceKVError) as e:
        c.advance([70, 0, 0] if c._n_free < 20 else [0, 70, 0])
    assert e.value.status == gk.GKV_ECAPACITY
    consistent()
    c.release(1)
    c.release(2)
    assert c._n_free == 40 and int(c.lens.sum()) == 0


def test_refusals(gk):
    K, V, lm = (t.cuda() for t in pool(1, 4, 16, 64, BF))
    table, lens = torch.zeros(1, 2, 2, 2, **I32), torch.ones(1, 2, 2, **I32)

    def make(**kw):
        a = dict(K=K, V=V, table=table, lens=lens, log_m=lm, Hq=4) | kw
        return gk.PagedCache(a.pop("K"), a.pop("V"), a.pop("table"), a.pop("lens"), **a)

    for kw, st in [(dict(V=V[:3].contiguous()), gk.GKV_EINVAL), (dict(V=V.float()), gk.GKV_EINVAL), (dict(Hq=3), gk.GKV_EINVAL),
                   (dict(lens=lens.long()), gk.GKV_EINVAL), (dict(log_m=lm[:2].contiguous()), gk.GKV_EINVAL),
                   (dict(Hq=18), gk.GKV_EUNSUPPORTED), (dict(K=K.half()), gk.GKV_EINVAL),
                   (dict(K=K[..., :32].contiguous(), V=V[..., :32].contiguous()), gk.GKV_EUNSUPPORTED)]:
        with pytest.raises(gk.GraceKVError) as e:
            make(**kw)
        assert e.value.status == st, kw
    with pytest.raises(ValueError):
        make(table=table.cpu())
    c = make()
    q, k, pos = torch.zeros(2, 4, 64, dtype=BF, device="cuda"), torch.zeros(2, 2, 64, dtype=BF, device="cuda"), torch.zeros(2, **I32)
    for call in (lambda: c.attention(1, q), lambda: c.attention(-1, q), lambda: c.attention(0, q[:1]), lambda: c.attention(0, q.float()),
                 lambda: c.append(1, k, k, pos), lambda: c.append(0, k[:1], k[:1], pos[:1]), lambda: c.append(0, k, k[:1], pos),
                 lambda: c.append(0, k, k, pos.long()), lambda: c.append(0, k.float(), k.float(), pos),
                 lambda: c.append(0, k, k, pos, cu_new=torch.zeros(2, **I32)), lambda: c.advance([1]), lambda: c.advance([1, -1]),
                 lambda: c.load_packed(2, k[0], k[0], None, torch.zeros(3, dtype=torch.int64, device="cuda")),
                 lambda: c.load_packed(0, k[0], k[0], None, torch.zeros(4, dtype=torch.int64, device="cuda"))):
        with pytest.raises(gk.GraceKVError) as e:
            call()
        assert e.value.status == gk.GKV_EINVAL
    for call in (lambda: c.load(0, None, 0), lambda: c.release(0)):
        with pytest.raises(gk.GraceKVError) as e:
            call()
        assert e.value.status == gk.GKV_ESTATE
    with pytest.raises(ValueError):
        c.attention(0, q.cpu())
    # log m for a cache that holds none; a rope base that is no base; pages that attention does not take
    with pytest.raises(gk.GraceKVError):
        make(log_m=None).load_packed(0, k[0], k[0], torch.zeros(2, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"))
    for base in (-1.0, math.nan, math.inf):
        with pytest.raises(gk.GraceKVError):
            make(rope_base=base).append(0, k, k, pos)
    K2 = torch.zeros(4, 24, 64, dtype=BF, device="cuda")
    with pytest.raises(gk.GraceKVError) as e:
        make(K=K2, V=K2.clone(), log_m=None).attention(0, q)
    assert e.value.status == gk.GKV_EUNSUPPORTED
    c.status()
