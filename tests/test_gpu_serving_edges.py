"""Serving operators where they can go wrong quietly: launches in a chain,
non-finite values that a sequence holds, bounds that do not fit, sizes past 32
bits, the branches that ordinary sizes do not take."""
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


# ---------------------------------------------------------------------- chains
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,d", [(1, 64), (7, 128), (64, 128)])
def test_in_place_rotation_and_attention_in_a_chain(gk, dtype, B, d):
    # One buffer of queries, rotated in place and attended by layer after layer without a wait: every
    # kernel starts under the end of the one that wrote what it reads.
    L, G, Hq, ps, n = 6, 2, 8, 32, 150
    g = torch.Generator(device="cuda").manual_seed(B)

    def normal(*shape):
        return torch.empty(*shape, dtype=dtype, device="cuda").normal_(generator=g)

    mp = -(-n // ps)
    table = torch.randperm(L * B * G * mp, device="cuda", generator=g).to(torch.int32).view(L, B, G, mp)
    pool = [normal(L * B * G * mp, ps, d) for _ in range(2)]
    k, v = (normal(L, B, G, d) for _ in range(2))
    q0, pos = normal(B, Hq, d), torch.randint(0, 100000, (B,), device="cuda", generator=g).to(torch.int32)

    def steps(wait):
        c = gk.PagedCache(pool[0].clone(), pool[1].clone(), table, torch.full((L, B, G), n, **I32), Hq=Hq, rope_base=1e4)
        q, seen = q0.clone(), []
        outs = torch.zeros(4 * L, B, Hq, d, dtype=dtype, device="cuda")
        torch.cuda.synchronize()
        for i in range(4 * L):
            l = i % L
            c.append(l, k[l], v[l], pos, q=q, out=q)
            if wait:
                torch.cuda.synchronize()
            c.attention(l, q, out=outs[i])
            if wait:
                torch.cuda.synchronize()
        c.status()
        return q, outs, c.K, c.V

    want = steps(True)
    for _ in range(3):
        for a, b in zip(steps(False), want):
            assert torch.equal(a, b)


# ------------------------------------------------------------- append's row bounds
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cu,bad", [([0, 2, 2, 5], False), ([0, 2, 2, 4], False), ([0, 5, 2, 5], True), ([0, 2, 9, 5], True),
                                    ([0, 2, 2, 9], True), ([-1, 2, 2, 5], True), ([0, 0, 0, 0], False)])
@pytest.mark.parametrize("tokens", [5, 3000])
def test_append_reports_bounds_that_do_not_fit(gk, cu, bad, dtype, tokens):
    # tokens past the last bound are of no request (a batch padded to a size): not stored, not reported
    G, ps, d = 2, 16, 64
    cu = [w * (tokens // 5) for w in cu]
    pages = -(-tokens * 2 // ps)
    g = torch.Generator(device="cuda").manual_seed(0)
    K, V = (torch.empty(3 * G * pages, ps, d, dtype=dtype, device="cuda").normal_(generator=g) for _ in range(2))
    table = torch.arange(3 * G * pages, **I32).view(1, 3, G, pages)
    lens = torch.full((1, 3, G), tokens * 2 - 3, **I32)
    k, v = (torch.empty(tokens, G, d, dtype=dtype, device="cuda").normal_(generator=g) for _ in range(2))
    c = gk.PagedCache(K, V, table, lens, Hq=G)
    before = K.clone()
    c.append(0, k, v, torch.zeros(tokens, **I32), cu_new=torch.tensor(cu, **I32))
    if bad:
        with pytest.raises(gk.GraceKVError) as e:
            c.status()
        assert e.value.status == gk.GKV_EINVAL
        return
    c.status()
    want = before.view(3, G, pages * ps, d)
    for b in range(3):
        n = cu[b + 1] - cu[b]
        want[b, :, tokens * 2 - 3 - n:tokens * 2 - 3] = k[cu[b]:cu[b + 1]].transpose(0, 1)
    assert torch.equal(K.view(3, G, pages * ps, d), want)


# --------------------------------------------------------------- the rotation's angle
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("base", [1.0, 1.0001, 2.0, 1e4, 5e5, 1e7])
def test_angles_at_every_size_of_position(gk, base, d):
    """Against exact turns.  The angle is off by 2^-26 turns (a fraction of 24 bits), 2^-32 (its upper word) and |p|
    times the stored turn's error, below 2^-53 (two powers, a product and a quotient in fp64 of a turn of at most
    1 / 2 pi); sine and cosine of it by 2^-23; a unit vector's rotation adds no rounding."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    two_pi = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534")
    pos = [0, 1, -1, 7, 4095, 131071, (1 << 20) + 1, (1 << 24) + 1, (1 << 27) - 1, 123456789, -987654321, (1 << 30) + 12345,
           (1 << 31) - 1, -(1 << 31)]
    x = torch.zeros(len(pos), 1, d, device="cuda")
    x[:, :, :d // 2] = 1.0
    K = torch.zeros(1, 16, d, device="cuda")
    c = gk.PagedCache(K, K.clone(), torch.zeros(1, 1, 1, 1, **I32), torch.tensor([[[len(pos)]]], **I32), Hq=1, rope_base=base)
    q = c.append(0, x, x, torch.tensor(pos, **I32), q=x, cu_new=torch.tensor([0, len(pos)], **I32))
    c.status()
    assert torch.equal(q[:, 0], K[0, :len(pos)])
    q = q[:, 0].double().cpu().numpy()
    for i in range(d // 2):
        turn = (Decimal(base).ln() * Decimal(-2 * i) / Decimal(d)).exp() / two_pi
        for t, p in enumerate(pos):
            a = 2 * math.pi * float((Decimal(p) * turn) % 1)
            tol = 2 * math.pi * (2.0 ** -26 + 2.0 ** -32 + abs(p) * 2.0 ** -53) + 2.0 ** -22
            assert abs(q[t, i] - math.cos(a)) <= tol and abs(q[t, i + d // 2] - math.sin(a)) <= tol, (i, p)

