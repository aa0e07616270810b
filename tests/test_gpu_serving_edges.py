"""Serving operators where they can go wrong quietly: launches in a chain,
non-finite values that a sequence holds, bounds that do not fit, sizes past 32
bits, the branches that ordinary sizes do not take."""
import math

import numpy as np
import pytest
import torch

from . import serving_reference as R
from .test_gpu_paged import append_case
from .test_gpu_prompt import check, cu, inputs

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


# ------------------------------------------------------- what ordinary sizes do not take
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [31, 32, 33, 64, 65, 300, 1100])
def test_prompts_of_many_sequences(gk, n, d, dtype):
    lens = [int(x) for x in np.random.default_rng(n).integers(0, 12, n)]
    lens[n // 2] = 200
    t = sum(lens)
    check(gk, *inputs(n, t, t, 4, 2, d, dtype), cu(lens), cu(lens))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [20, 40, 70])
def test_many_sequences_whose_keys_are_split(gk, n, dtype):
    # one or two queries each over a few thousand keys, one sequence with none
    rng = np.random.default_rng(n)
    nq, nk = rng.integers(1, 3, n), rng.integers(1000, 2500, n)
    nk[3] = 0
    nq[5] = 0
    check(gk, *inputs(n, int(nq.sum()), int(nk.sum()), 4, 1, 64, dtype), cu(nq.tolist()), cu(nk.tolist()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["query token", "query head", "key token", "value token"])
@pytest.mark.parametrize("nq,nk", [(200, 200), (3, 4000), (70, 900)])
def test_bf16_tensors_without_a_tensor_map(gk, nq, nk, which, d):
    # an axis broadcast by a zero stride has no tensor map: these run on CUDA cores, whole and in parts
    q, k, v = (t.cuda() for t in inputs(nq, nq, nk, 8, 2, d, BF))
    if which == "query token":
        q = q[:1].expand(nq, 8, d)
    elif which == "query head":
        q = q[:, :1].expand(nq, 8, d)
    elif which == "key token":
        k = k[:1].expand(nk, 2, d)
    else:
        v = v[:1].expand(nk, 2, d)
    check(gk, q, k, v, cu([nq]), cu([nk]))
    lens = [1, 0, nq - 1]
    keys = [0, 5, nk - 5]
    check(gk, q, k, v, cu(lens), cu(keys))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_rows_past_2_31_elements(gk, d, dtype):
    # tokens 2^24 elements apart: the last rows begin past 2^31 elements (and 2^32 bytes)
    n, Hq, G = 180, 4, 2
    buf = torch.empty(n, 1 << 24, dtype=dtype, device="cuda")
    q, k, v = inputs(n, n, n, Hq, G, d, dtype)
    at, views = 1 << 23, []
    for t in (q, k, v, q):
        w = t.shape[1] * d
        views.append(buf[:, at:at + w].view(n, t.shape[1], d))
        at += w
    for view, t in zip(views, (q, k, v)):
        view.copy_(t)
    c = torch.tensor([0, 100, n], **I32)
    op = gk.PromptAttention(G=G, Hq=Hq, d=d, dtype=dtype)
    op(*views[:3], c, out=views[3])
    op.status()
    assert torch.equal(views[3], op(q.cuda(), k.cuda(), v.cuda(), c))
    for view, t in zip(views, (q, k, v)):
        assert torch.equal(view.cpu(), t)                   # nothing was written beside the output
    del buf, views
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,S", [(BF, 128), (F32, 64)])
def test_attention_over_more_tiles_than_32_bits_hold_products_of(gk, dtype, S):
    """4.3 million tiles, of a few pages that the tables name again and again.  All logits are 0 and all values 1, 0 or -1,
    so that every sum is a whole number that fp32 holds exactly: one entry too many or too few shows."""
    ps, d = 4096, 64
    m = (540 if dtype == BF else 530) // 2 * 2              # pages of a sequence
    K, V = torch.zeros(2, ps, d, dtype=dtype, device="cuda"), torch.ones(2, ps, d, dtype=dtype, device="cuda")
    V[1, :, 0] = -1                                         # channel 0: pages cancel; 1: one page of two; others: 1
    V[1, :, 1] = 0
    table = (torch.arange(m, device="cuda") % 2).to(torch.int32).repeat(S, 1).view(1, S // 2, 2, m).contiguous()
    lens = torch.full((1, S // 2, 2), m * ps, **I32)
    lens[0, 5] = torch.tensor([0, 2 * ps], **I32)
    lens[0, 7, 1] = m * ps - 2 * ps
    tile = 64 if dtype == BF else 32
    assert int(lens.long().sum()) // tile > 1 << 22
    c = gk.PagedCache(K, V, table, lens, Hq=4)
    q = torch.randn(S // 2, 4, d, device="cuda").to(dtype)
    out = c.attention(0, q)
    c.status()
    want = torch.ones(S // 2, 4, d, dtype=dtype, device="cuda")
    want[..., 0], want[..., 1] = 0, 0.5
    want[5, :2] = 0
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_append_of_many_tokens_to_several_requests(gk, d, dtype):
    # four rows a thread, rows that do not divide by four
    counts = [1500, 0, 900, 1]
    append_case(gk, counts, [[0, 3, 7]] * 4, 48, 9, 3, d, dtype, 5e5, np.arange(2401) * 7, strided=True)
    append_case(gk, counts, [[0, 3, 7]] * 4, 48, 6, 3, d, dtype, 0.0, np.arange(2401), with_q=False)
