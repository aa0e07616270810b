"""Attention over quantised shared prefixes whose rows have scales of all sizes: the same softmax as over the values that
the rows stand for, as gracekv_quant_attention computes it."""
import math

import numpy as np
import pytest
import torch

from . import serving_reference as R
from .test_gpu_quant_attention import junk, pages, real
from .test_gpu_shared import BF, F32, expected, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


class Side:
    """A quantised cache; edit(K, ks, V, vs, lm) changes pool rows and may return those that have no weight, which, like
    entries of log m = -inf, count 0 in `rows`."""

    def __init__(self, gk, lens, ps, Hq, d, dtype, seed, edit):
        lens = np.asarray(lens)
        self.table, n = R.scattered_table(np.random.default_rng(seed), lens, ps)
        ((K, ks), (V, vs)), lm = pages(seed, n, ps, d, spread=2.0)
        at = junk(self.table, lens, ps, n)
        none = edit(K, ks, V, vs, lm)
        self.K, self.V, self.lm, self.lens = real(K, ks), real(V, vs), lm.clone(), lens
        if none is not None:
            self.lm.view(-1)[none] = -math.inf
        for t in (self.K, self.V):
            t[self.lm == -math.inf] = 0
        for t in (K, V):
            t.view(torch.uint8)[at] = 0x7f
        for t in (ks, vs):
            t[at] = 255
        lm[at] = math.nan
        self.cache = gk.PagedCache(K.cuda(), V.cuda(), self.table.cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), Hq=Hq,
                                   log_m=lm.cuda(), k_scale=ks.cuda(), v_scale=vs.cuda(), dtype=dtype)

    def rows(self, i):
        n = int(self.lens[i])
        return tuple(R.entries(t, self.table[i], n).double() for t in (self.K, self.V, self.lm))


def attend(gk, edit, dtype, d, B, q_scale, seed, n=700, first=None, q=None):
    rng = np.random.default_rng(seed)
    own, pre = rng.integers(0, 40, (1, B, 2)), np.array([[[n, n - 5]]])
    a, p = Side(gk, own, 16, 8, d, dtype, seed, edit), Side(gk, pre, 32, 8, d, dtype, seed + 100, edit)
    if q is None:
        q = queries(B, 8, d, dtype, seed + 1, q_scale)
    if first is not None:
        q[..., 0] = first
    f = gk.SharedAttention(a.cache, p.cache)
    out = f(0, q.cuda()).double().cpu()
    f.status()
    want, tol = expected(q, a, p, [0, B])
    assert torch.isfinite(out).all()
    assert ((out - want).abs() <= tol).all(), f"{float(((out - want).abs() - tol).max()):.3e} over its bound"


def no_zeros(K, ks, V, vs, lm):
    zero = (K.view(torch.uint8) == 0).all(-1)
    K.view(torch.uint8)[zero] = 0x31
    ks[zero] = 120


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [6, 17, 64, 127, 128, 129, 300, 1000])
def test_keys_of_one_size(gk, dtype, d, n):
    # scales close together, queries of ordinary size: log m is a part of the product
    attend(gk, no_zeros, dtype, d, 3, 1.0, n, n=n)
    attend(gk, no_zeros, dtype, d, 70, 1.0, n, n=n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 70])
def test_tiles_of_both_kinds(gk, d, B):
    # some tiles of scales close together, some not, and row tiles of ordinary and of large queries on them
    def keys(K, ks, V, vs, lm):
        no_zeros(K, ks, V, vs, lm)
        ks.view(-1)[5::301] = 7

    attend(gk, keys, BF, d, B, 1.0, 15, n=3000)

    def some(K, ks, V, vs, lm):
        keys(K, ks, V, vs, lm)
        lm.view(-1)[::7] = -math.inf
    q = queries(B, 8, d, BF, 17)
    q[:2] *= 2.0 ** -40                      # their logits are log m but for 2^-30
    q[2:, 5] = 0
    attend(gk, some, BF, d, B, 1.0, 16, n=3000, q=q)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("by", [-100, -90, -60, -45, 45, 60, 90])
def test_keys_of_all_sizes(gk, dtype, d, B, by):
    # small keys with large queries and the other way round: the same logits
    def keys(K, ks, V, vs, lm):
        ks.copy_((ks.int() + by).clamp(7, 246).to(torch.uint8))

    attend(gk, keys, dtype, d, B, 2.0 ** -by, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("by", [14, 17, 25, 50, 80])
def test_small_keys_beside_large_ones(gk, dtype, d, B, by):
    # keys 2^by times as large as the others in some tiles, all against every query: they have no weight (logits of
    # -2^(by + 8) / sqrt(d)), and the others' logits differ as they did
    def keys(K, ks, V, vs, lm):
        big = torch.zeros(lm.numel(), dtype=torch.bool)
        big[17::190] = True
        codes = K.view(torch.uint8).view(-1, d)
        codes[big] = 0
        codes[big, 0] = 0xf8                 # -256
        ks.view(-1)[big] = 127 + by
        return big

    attend(gk, keys, dtype, d, B, 1.0, 2, first=1.0)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [3, 40])
def test_both_ends_of_the_scales(gk, dtype, B):
    # the largest ones without weight; the smallest ones' keys and values are next to nothing (fp32 logits below 2^100)
    def keys(K, ks, V, vs, lm):
        ks.view(-1)[::4] = 7
        ks.view(-1)[1::4] = 246
        lm.view(-1)[1::4] = -math.inf

    attend(gk, keys, dtype, 128, B, 1.0 if dtype == BF else 2.0 ** -27, 3)

    def values(K, ks, V, vs, lm):
        vs.view(-1)[::3] = 7
        vs.view(-1)[1::3] = 246
        lm.view(-1)[1::3] = -math.inf
    attend(gk, values, dtype, 64, B, 1.0, 4)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("by", [-100, 100])
def test_values_of_all_sizes(gk, dtype, B, by):
    # the outputs' size, and a last tile whose values are far larger: what was summed before is scaled down beside them
    def all_of(K, ks, V, vs, lm):
        vs.copy_((vs.int() + by).clamp(7, 246).to(torch.uint8))

    rng = np.random.default_rng(5)
    own, pre = rng.integers(0, 40, (1, B, 2)), np.array([[[700, 695]]])
    a, p = Side(gk, own, 16, 8, 64, dtype, 5, all_of), Side(gk, pre, 32, 8, 64, dtype, 105, all_of)
    q = queries(B, 8, 64, dtype, 6)
    f = gk.SharedAttention(a.cache, p.cache)
    out = f(0, q.cuda()).double().cpu()
    f.status()
    one = 2.0 ** by
    for s in (a, p):
        s.V = s.V / one
    want, tol = expected(q, a, p, [0, B])
    assert ((out / one - want).abs() <= tol).all()


@pytest.mark.parametrize("B", [3, 40])
def test_a_late_tile_of_larger_values(gk, B):
    def late(K, ks, V, vs, lm):
        vs[-6:] += 12                        # scattered over the tiles by the table, each piece meets some of them late
    attend(gk, late, BF, 128, B, 1.0, 7, n=3000)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_length_past_the_table(gk, dtype):
    # is cut there and reported: the entries that the table leads to count
    own, pre = np.array([[[9, 4], [0, 30]]]), np.array([[[96, 64]]])
    a, p = Side(gk, own, 16, 8, 64, dtype, 12, lambda *x: None), Side(gk, pre, 32, 8, 64, dtype, 13, lambda *x: None)
    q = queries(2, 8, 64, dtype, 14)
    f = gk.SharedAttention(a.cache, p.cache)
    p.cache.lens[0, 0, 0] = 96 + 777
    out = f(0, q.cuda()).double().cpu()
    with pytest.raises(gk.GraceKVError) as e:
        f.status()
    assert e.value.status == gk.GKV_EINVAL
    want, tol = expected(q, a, p, [0, 2])
    assert ((out - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
@pytest.mark.parametrize("way", ["some", "first", "last"])
def test_large_rows_under_masks(gk, dtype, d, B, way):
    # keys and values of any size under the lowest log m are as if they were not there: scattered, before all others of a
    # sequence, behind them
    low = torch.finfo(torch.float32).min
    lens = np.array([[[900, 895]]])
    table, n = R.scattered_table(np.random.default_rng(20), lens, 32)
    out = torch.zeros(n * 32, dtype=torch.bool)
    for h in range(2):
        e = torch.arange(int(lens[0, 0, h]))
        at = table[0, 0, h, e // 32].long() * 32 + e % 32
        out[at[{"some": e % 7 == 3, "first": e < 300, "last": e >= 300}[way]]] = True

    def edit(K, ks, V, vs, lm):
        if lm.numel() != out.numel():
            return None
        vs.view(-1)[out] = 230
        ks.view(-1)[out] += 3
        lm.view(-1)[out] = low
        return out

    own = Side(gk, np.random.default_rng(21).integers(0, 40, (1, B, 2)), 16, 8, d, dtype, 22, lambda *a: None)
    pre = Side(gk, lens, 32, 8, d, dtype, 20, edit)
    assert torch.equal(pre.table, table)
    q = queries(B, 8, d, dtype, 23)
    f = gk.SharedAttention(own.cache, pre.cache)
    got = f(0, q.cuda()).double().cpu()
    f.status()
    want, tol = expected(q, own, pre, [0, B])
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= tol).all(), f"{float(((got - want).abs() - tol).max()):.3e} over its bound"
