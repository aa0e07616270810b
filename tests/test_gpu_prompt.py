"""The prompt's attention: CUDA path (gracekv_prompt_*) against its definition
in 64 bits (serving_reference.prompt, which also derives the tolerances)."""
import math

import pytest
import torch

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


def cu(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


def inputs(seed, nq, nk, Hq, G, d, dtype, sharp=3.0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(nq, Hq, d, generator=g)
    q[:, 1::2] *= sharp
    return tuple(t.to(dtype) for t in (q, torch.randn(nk, G, d, generator=g), torch.randn(nk, G, d, generator=g)))


def check(gk, q, k, v, cq, ck, op=None, **kw):
    Hq, G, d = q.shape[1], k.shape[1], q.shape[2]
    op = op or gk.PromptAttention(G=G, Hq=Hq, d=d, dtype=q.dtype)
    i32 = dict(dtype=torch.int32, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    op(q.cuda() if not q.is_cuda else q, k.cuda() if not k.is_cuda else k, v.cuda() if not v.is_cuda else v,
       torch.tensor(cq, **i32), torch.tensor(ck, **i32), out=out, lse=lse, return_lse=True, **kw)
    op.status()
    want, wlse, tol, ltol = R.prompt(q, k, v, cq, ck, bf16=q.dtype == BF)
    got, glse = out.double().cpu(), lse.double().cpu()
    none = torch.isnan(wlse)                       # rows of no sequence keep what was there
    assert (got[none] == 7.0).all() and (glse[none] == 7.0).all()
    empty = torch.isinf(wlse)
    assert (got[empty] == 0).all() and torch.equal(glse[empty], wlse[empty])
    rest = ~none & ~empty
    err, lerr = (got - want).abs()[rest], (glse - wlse).abs()[rest]
    assert torch.isfinite(got[rest]).all()
    assert (err <= tol[rest]).all(), f"out {float((err - tol[rest]).max()):.3e} over its bound"
    assert (lerr <= ltol[rest]).all(), f"lse {float((lerr - ltol[rest]).max()):.3e} over its bound"
    return out, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 400])
def test_one_sequence(gk, dtype, d, n):
    check(gk, *inputs(n, n, n, 4, 2, d, dtype), cu([n]), cu([n]))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,G", [(1, 1), (6, 3), (6, 2), (4, 1), (10, 2), (6, 1), (14, 2), (8, 1), (32, 8)])
def test_head_layouts(gk, dtype, Hq, G):
    lens = [70, 1, 200]
    check(gk, *inputs(Hq, 271, 271, Hq, G, 64, dtype), cu(lens), cu(lens))
    check(gk, *inputs(Hq, 271, 271, Hq, G, 128, dtype), cu(lens), cu(lens))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_packed_with_empty_sequences(gk, dtype, d):
    lens = [0, 5, 0, 130, 1, 0, 0, 64, 257, 33, 0]
    n = sum(lens)
    check(gk, *inputs(3, n, n, 4, 2, d, dtype), cu(lens), cu(lens))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_that_continue_a_prompt(gk, dtype, d):
    # more keys than queries; fewer (the first queries see nothing); no key at all; one query over many keys
    nq, nk = [5, 130, 40, 7, 1, 1, 64, 100], [300, 131, 12, 0, 1000, 1, 65, 640]
    check(gk, *inputs(4, sum(nq), sum(nk), 8, 2, d, dtype), cu(nq), cu(nk))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nq,nk", [(1, 5000), (3, 4097), (17, 9000), (130, 2500)])
def test_few_queries_over_a_long_axis(gk, dtype, nq, nk):
    check(gk, *inputs(5, nq, nk, 8, 2, 128, dtype), cu([nq]), cu([nk]))
    check(gk, *inputs(6, nq, nk, 4, 1, 64, dtype), cu([nq]), cu([nk]))


@pytest.mark.parametrize("nq,nk,G", [(3, 12000, 80), (300, 6000, 20), (70, 9000, 1)])
def test_parts_of_many_and_of_few_blocks(gk, nq, nk, G):
    check(gk, *inputs(25, nq, nk, G, G, 64, BF), cu([nq]), cu([nk]))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_outside_the_sequences_do_not_matter(gk, dtype, d):
    # NaN and infinity in the rows before, after and between the keys' sequences
    q, k, v = inputs(7, 400, 500, 4, 2, d, dtype)
    cq, ck = [3, 73, 73, 303], [50, 120, 120, 350]
    for lo, hi in ((0, 50), (350, 500)):
        k[lo:hi] = math.nan
        v[lo:hi] = math.inf
        v[lo + 1:hi:2] = math.nan
    check(gk, q, k, v, cq, ck)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_neighbouring_sequences_do_not_matter(gk, dtype):
    # a non-finite sequence leaves the others as they are
    lens = [100, 77, 140]
    n = sum(lens)
    q, k, v = inputs(8, n, n, 4, 2, 128, dtype)
    clean = check(gk, q, k, v, cu(lens), cu(lens))[0]
    k[100:177] = math.nan
    v[100:177] = math.inf
    q[100:177] = -math.inf
    i32 = dict(dtype=torch.int32, device="cuda")
    op = gk.PromptAttention(G=2, Hq=4, d=128, dtype=dtype)
    out = op(q.cuda(), k.cuda(), v.cuda(), torch.tensor(cu(lens), **i32))
    op.status()
    assert torch.equal(out[:100], clean[:100]) and torch.equal(out[177:], clean[177:])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_strides(gk, dtype, d):
    n, Hq, G = 150, 6, 2
    q, k, v = inputs(9, n, n, Hq, G, d, dtype)
    fused = torch.cat([t.reshape(n, -1) for t in (q, k, v)], 1).cuda()
    qs, ks, vs = (t.view(n, -1, d) for t in fused.split([Hq * d, G * d, G * d], 1))
    a, _ = check(gk, qs, ks, vs, cu([n]), cu([n]))
    # head-major keys and values, as the compressor takes them
    kt, vt = (t.cuda().transpose(0, 1).contiguous().transpose(0, 1) for t in (k, v))
    b, _ = check(gk, q, kt, vt, cu([n]), cu([n]))
    assert torch.equal(a, b)
    # head-major queries and outputs, through the strided output
    op = gk.PromptAttention(G=G, Hq=Hq, d=d, dtype=dtype)
    qt = q.cuda().transpose(0, 1).contiguous().transpose(0, 1)
    ot = torch.empty(Hq, n, d, dtype=dtype, device="cuda").transpose(0, 1)
    op(qt, kt, vt, torch.tensor([0, n], dtype=torch.int32, device="cuda"), out=ot)
    assert torch.equal(ot, a)
    # one shared key head broadcast to all groups by a zero stride
    k1, v1 = (t[:, :1].cuda().expand(n, G, d) for t in (k, v))
    check(gk, q, k1, v1, cu([n]), cu([n]))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_logits(gk, dtype):
    # logits of several hundred: the running maximum keeps the exponentials in range
    n = 300
    q, k, v = inputs(10, n, n, 4, 2, 64, dtype, sharp=60.0)
    check(gk, q, k, v, cu([n]), cu([n]))
    check(gk, -q.abs(), k.abs(), v, cu([n]), cu([n]))     # all of them far below 0


@pytest.mark.parametrize("fall", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [95, 96, 97, 128, 129, 192, 193, 288, 300, 577])
def test_logits_that_rise_or_fall_along_the_keys(gk, n, d, fall):
    """Every key tile raises the rows' maxima by far more than the one before
    left (or none does after the first), the last tile of a row too."""
    q, k, v = inputs(23, n, n, 8, 2, d, torch.float32, sharp=1.0)
    u = torch.ones(d)
    q, k = q * 0.1 + u, k * 0.1
    t = torch.arange(n).flip(0) if fall else torch.arange(n)
    k = k + (0.15 * t / math.sqrt(d))[:, None, None] * u            # 0.15 a key in the scaled product
    check(gk, q.to(BF), k.to(BF), v.to(BF), cu([n]), cu([n]))


def test_results_do_not_depend_on_timing(gk):
    lens = [513, 100, 1, 900]
    n = sum(lens)
    for dtype in (BF, F32):
        q, k, v = (t.cuda() for t in inputs(11, n, n, 8, 2, 128, dtype))
        c = torch.tensor(cu(lens), dtype=torch.int32, device="cuda")
        op = gk.PromptAttention(G=2, Hq=8, d=128, dtype=dtype)
        first = op(q, k, v, c, return_lse=True)
        for _ in range(5):
            again = op(q, k, v, c, return_lse=True)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_one_call_after_another_of_other_shapes(gk):
    # one object, its workspace reused by calls of every shape without a wait between them
    op = gk.PromptAttention(G=2, Hq=8, d=128, dtype=BF)
    jobs = []
    for i, (nq, nk) in enumerate([(1, 6000), (300, 300), (5, 3000), (0, 10), (700, 900), (1, 1)]):
        q, k, v = inputs(20 + i, nq, nk, 8, 2, 128, BF)
        c = [torch.tensor([0, m], dtype=torch.int32, device="cuda") for m in (nq, nk)]
        jobs.append((q, k, v, nq, nk, op(q.cuda(), k.cuda(), v.cuda(), *c)))
    op.status()
    for q, k, v, nq, nk, out in jobs:
        want, _, tol, _ = R.prompt(q, k, v, [0, nq], [0, nk], bf16=True)
        assert ((out.double().cpu() - want).abs() <= tol).all()


def test_another_stream(gk):
    s = torch.cuda.Stream()
    q, k, v = (t.cuda() for t in inputs(12, 260, 260, 4, 2, 64, BF))
    c = torch.tensor([0, 260], dtype=torch.int32, device="cuda")
    op = gk.PromptAttention(G=2, Hq=4, d=64, dtype=BF)
    here = op(q, k, v, c)
    s.wait_stream(torch.cuda.current_stream())
    there = op(q, k, v, c, stream=s)
    op.status(s)
    assert torch.equal(here, there)


def test_made_here_and_used_on_another_stream(gk):
    # the current stream is another one from the first call on; the object goes while its work is queued
    q, k, v = (t.cuda() for t in inputs(17, 400, 400, 8, 2, 64, BF))
    c = torch.tensor([0, 400], dtype=torch.int32, device="cuda")
    want = gk.PromptAttention(G=2, Hq=8, d=64, dtype=BF)(q, k, v, c)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        op = gk.PromptAttention(G=2, Hq=8, d=64, dtype=BF)
        first = op(q, k, v, c)
    op2 = gk.PromptAttention(G=2, Hq=8, d=64, dtype=BF)
    with torch.cuda.stream(s):
        second = op2(q, k, v, c)
    del op, op2
    s.synchronize()
    assert torch.equal(first, want) and torch.equal(second, want)


def test_graph_capture(gk):
    q, k, v = (t.cuda() for t in inputs(13, 300, 300, 4, 2, 128, BF))
    c = torch.tensor([0, 120, 300], dtype=torch.int32, device="cuda")
    op = gk.PromptAttention(G=2, Hq=4, d=128, dtype=BF)
    out = torch.empty_like(q)
    want = op(q, k, v, c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op(q, k, v, c, out=out)
    out.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cq,ck", [([0, 50, 40, 90], [0, 50, 60, 90]), ([0, 50, 120], [0, 50, 100]),
                                   ([0, 50, 90], [0, 50, 101]), ([-4, 20, 40], [0, 20, 40]),
                                   ([0, 20, 40], [0, -3, 40]), ([0, 30, 60], [10, 5, 40])])
def test_bounds_that_do_not_fit_are_reported(gk, dtype, cq, ck):
    q, k, v = (t.cuda() for t in inputs(14, 100, 100, 4, 2, 64, dtype))
    op = gk.PromptAttention(G=2, Hq=4, d=64, dtype=dtype)
    op(q, k, v, *(torch.tensor(c, dtype=torch.int32, device="cuda") for c in (cq, ck)))
    with pytest.raises(gk.GraceKVError) as e:
        op.status()
    assert e.value.status == gk.GKV_EINVAL
    op.status()                                   # cleared; the object works on
    check(gk, *inputs(15, 40, 40, 4, 2, 64, dtype), [0, 40], [0, 40], op=op)


def test_empty_calls(gk):
    op = gk.PromptAttention(G=2, Hq=4, d=64, dtype=BF)
    i32 = dict(dtype=torch.int32, device="cuda")
    z = torch.zeros(0, 4, 64, dtype=BF, device="cuda")
    k = torch.zeros(0, 2, 64, dtype=BF, device="cuda")
    assert op(z, k, k, torch.tensor([0], **i32)).shape == (0, 4, 64)
    out, lse = op(z.new_ones(3, 4, 64), k, k, torch.tensor([0, 3], **i32), torch.tensor([0, 0], **i32), return_lse=True)
    op.status()
    assert (out == 0).all() and torch.isinf(lse).all()


def test_refusals(gk):
    i32 = dict(dtype=torch.int32, device="cuda")
    q, k, v = (t.cuda() for t in inputs(16, 10, 10, 4, 2, 64, BF))
    c = torch.tensor([0, 10], **i32)
    op = gk.PromptAttention(G=2, Hq=4, d=64, dtype=BF)
    bad = [(q.float(), k, v, c), (q, k.float(), v, c), (q[:, :3], k, v, c), (q, k[:9], v, c), (q, k, v[..., :32], c),
           (q, k, v, c.long()), (q.transpose(0, 2).contiguous().transpose(0, 2), k, v, c)]
    for args in bad:
        with pytest.raises(gk.GraceKVError) as e:
            op(*args)
        assert e.value.status == gk.GKV_EINVAL
    with pytest.raises(ValueError):
        op(q.cpu(), k, v, c)
    odd = torch.zeros(10 * 4 * 64 + 4, dtype=BF, device="cuda")[4:].view(10, 4, 64)       # 8 bytes off
    with pytest.raises(gk.GraceKVError):
        op(odd, k, v, c)
    ragged = torch.zeros(10, 4 * 64 + 4, dtype=BF, device="cuda")[:, :256].view(10, 4, 64)   # rows 8 bytes off
    with pytest.raises(gk.GraceKVError):
        op(ragged, k, v, c)
    for kw, st in [(dict(G=2, Hq=4, d=96), gk.GKV_EUNSUPPORTED), (dict(G=2, Hq=5, d=64), gk.GKV_EINVAL),
                   (dict(G=1, Hq=9, d=64), gk.GKV_EUNSUPPORTED)]:
        with pytest.raises(gk.GraceKVError) as e:
            gk.PromptAttention(dtype=BF, **kw)
        assert e.value.status == st
    with pytest.raises(gk.GraceKVError):
        gk.PromptAttention(G=2, Hq=4, d=64, dtype=torch.float16)
