"""What the softmax weights of a shared prefix keep of themselves for the value product."""
import math

import pytest
import torch

from . import quant_reference as Q
from .test_gpu_shared import BF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


def opposed(gk, n, B, d, quant, bits):
    """Outputs over a prefix, and over the same entries as a request's own, where nearly equal weights to either side of
    the middle between two numbers of `bits` bits have opposite values: rounded once they no longer cancel.
    Every eighth entry has weight 1 and the value 0, so that the others lie between 1/2 and 1."""
    i = torch.arange(n)
    middle = 0.75 + 2.0 ** -(bits + 1)
    p = torch.where(i % 2 == 0, middle - 2.0 ** -(bits + 5), middle + 2.0 ** -(bits + 5)).double()
    p[i % 8 == 0] = 1.0
    sign = torch.where(i % 2 == 0, 1.0, -1.0)
    sign[i % 8 == 0] = 0.0
    lm = torch.log(p).float()
    V = sign[:, None] * torch.linspace(1, 1.75, 4).repeat(d // 4)[None]          # exact in every type
    K = torch.zeros(n, d)
    pages = -(-n // 64)

    def room(x):
        return torch.cat([x, torch.zeros(pages * 64 - n, *x.shape[1:])]).view(pages, 64, *x.shape[1:])
    sc = {}
    if quant:
        (Kc, ks), (Vc, vs) = Q.pool(K), Q.pool(V)
        Kp, Vp = room(Kc.float()).to(torch.float8_e4m3fn), room(Vc.float()).to(torch.float8_e4m3fn)
        sc = dict(k_scale=room(ks.float()).to(torch.uint8).cuda(), v_scale=room(vs.float()).to(torch.uint8).cuda(), dtype=BF)
    else:
        Kp, Vp = room(K).to(BF), room(V).to(BF)
    i32 = dict(dtype=torch.int32, device="cuda")

    def cache(B, table, n):
        return gk.PagedCache(Kp.cuda(), Vp.cuda(), table, torch.full((1, B, 1), n, **i32), Hq=4, log_m=room(lm).cuda(), **sc)
    pre = cache(1, torch.arange(pages, **i32).view(1, 1, 1, pages), n)
    own = cache(B, torch.full((1, B, 1, 1), -1, **i32), 0)
    q = torch.ones(B, 4, d, dtype=BF, device="cuda")
    f = gk.SharedAttention(own, pre)
    out = f(0, q).double().cpu()
    f.status()
    w = torch.softmax(lm.double(), 0)
    want, sure = w @ V.double(), w @ V.double().abs()
    alone = pre.attention(0, q[:1]).double().cpu()
    return out, alone, want, sure


def bound(want, sure, n, keeps):
    """Weights that keep `keeps` bits, their exponentials and log m 2^-21 off, n fp32 sums of values below 2 over the sum
    of weights of at least n / 2, the output's rounding."""
    return (2.0 ** -keeps + 2 * 2.0 ** -21) * sure + 2.0 ** -24 * (n + 64) + 2.0 ** -8 * want.abs()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
def test_bf16_weights_keep_16_bits(gk, d, B):
    # n of a tile and a half, and of several pieces
    for n in (200, 1500):
        out, alone, want, sure = opposed(gk, n, B, d, False, 8)
        tol = bound(want, sure, n, 16)
        assert ((alone - want).abs() <= tol).all()
        assert ((out - want).abs() <= tol).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [3, 40])
def test_f16_weights_keep_11_bits(gk, d, B):
    # over quantised pages; those of one request's own pages keep 22
    for n in (200, 1500):
        out, alone, want, sure = opposed(gk, n, B, d, True, 11)
        assert ((alone - want).abs() <= bound(want, sure, n, 22)).all()
        assert ((out - want).abs() <= bound(want, sure, n, 11)).all()
