"""The angle of quantised keys, by keys whose exact value lies next to the middle between two codes: which code they get
tells the cosine to 2^-22 of itself."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
MARGIN = 2.0 ** -22


@pytest.fixture(scope="module", autouse=True)
def gk():
    import __graft_entry__ as g
    g.build()
    assert torch.cuda.is_available()
    from paper_2608_07001_gb300 import gracekv
    return gracekv


def keys(rng, N, d, base):
    """(x [N, d] fp32, pos [N], wanted [N, d / 2], chosen): rows whose pair 0 makes 2^0 the scale (a largest value of 283 to
    400) and whose pairs i have x[i] cos(phi_i) within 2 to 4 MARGIN / 2 above or below the middle of two codes, x[i + d / 2] = 0.

    The kernel's cosine is within 1.4 of a float's last bit, at most 1.4 2^-23 of itself; the product rounds once (2^-24);
    the angle is off by 2^-33 turns and less than |pos| 2^-53, which tan(phi) < 16 makes 2^-26 of the cosine: 0.99
    MARGIN together."""
    half = d // 2
    pos = rng.integers(1, 1 << 17, N)
    phi = pos[:, None] * base ** (-2.0 * np.arange(half) / d)
    c = np.cos(phi)
    step = 2.0 ** -3
    k = rng.integers(0, 8, (N, half))                       # codes 1 + k / 8, scaled
    size = np.floor(np.log2(np.abs(c))) + rng.integers(0, 7, (N, half))
    middle = (1 + (k + 0.5) * step) * 2.0 ** size
    up = rng.integers(0, 2, (N, half)) * 2 - 1
    target = middle * (1 + up * MARGIN * rng.uniform(1.25, 2.0, (N, half)))
    x = np.zeros((N, d), np.float32)
    x[:, :half] = (target / c).astype(np.float32)
    x[:, 0] = 400.0
    got = x[:, :half].astype(np.float64) * c                # rounding x moved it by 2^-24
    off = got / middle - 1
    s = np.abs(np.sin(phi))
    chosen = (np.abs(off) >= MARGIN) & (np.abs(off) < 4 * MARGIN) & (np.abs(c) > 1 / 16) & (np.abs(x[:, :half]) <= 400)
    chosen &= (np.abs(x[:, :half]) * s <= 400)
    chosen[:, 0] = False
    x[:, 1:half][~chosen[:, 1:]] = 0
    lower = (1 + k * step) * 2.0 ** size
    wanted = np.where(off > 0, lower + step * 2.0 ** size, lower)
    return x, pos, wanted, chosen


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("base", [1e4, 5e5])
def test_codes_next_to_a_middle(gk, d, base):
    rng = np.random.default_rng(d)
    N = 4000
    x, pos, wanted, chosen = keys(rng, N, d, base)
    assert chosen.sum() > N * d // 16
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = -(-N // 64)
    pool = [torch.empty(pages, 64, d, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    scale = [torch.empty(pages, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c = gk.PagedCache(*pool, torch.arange(pages, **i32).view(1, 1, 1, pages), torch.full((1, 1, 1), N, **i32), Hq=1, rope_base=base,
                      k_scale=scale[0], v_scale=scale[1], dtype=torch.float32)
    k = torch.from_numpy(x).cuda().view(N, 1, d)
    c.append(0, k, k, torch.from_numpy(pos.astype(np.int32)).cuda(), cu_new=torch.tensor([0, N], **i32))
    c.status()
    assert (scale[0].view(-1)[:N] == 127).all()
    got = pool[0].float().view(-1, d)[:N, :d // 2].double().cpu().numpy()
    # sizes below 2^-6 have the codes' least step, a grid of their own
    normal = chosen & (np.abs(wanted) >= 2.0 ** -6)
    assert np.array_equal(got[normal], wanted[normal])
