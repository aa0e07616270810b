"""Row bounds of the prompt's attention that do not fit: the sequences that do are
computed all the same, the others are left alone and reported."""
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


def computed(cq, ck, n_q, n_k):
    """The sequences that are computed: bounds that ascend within the rows, queries
    that do not begin below the end of an earlier such sequence."""
    end, s = 0, []
    for i, (a, b, c, e) in enumerate(zip(cq[:-1], cq[1:], ck[:-1], ck[1:])):
        if 0 <= a <= b <= n_q:
            if a >= end and 0 <= c <= e <= n_k:
                s.append(i)
            end = max(end, b)
    return s


def ascending(lens, first=0):
    return [first + int(n) for n in np.concatenate([[0], np.cumsum(lens)])]


MANY = ascending([7, 1, 0, 30] * 11)
CROWD = ascending([1, 0] * 510 + [3] * 24)
THRONG = ascending([1, 0] * 520 + [5] * 20)
CASES = [
    # (cu_q, cu_k, sequences that are left out)
    ([0, 1000, 200, 900], [0, 1000, 1010, 1500], [1, 2]),
    ([0, 300, 100, 250, 300, 420], [0, 300, 310, 460, 510, 630], [1, 2, 3]),
    ([0, 100, 50, 100, 260], [0, 100, 130, 180, 340], [1, 2]),
    ([0, 100, 5000, 100, 260], [0, 100, 130, 180, 340], [1, 2]),
    ([0, 100, -7, 100, 260], [0, 100, 130, 180, 340], [1, 2]),
    ([2000, 0, 130, 260], [0, 10, 140, 270], [0]),
    ([200, 0, 130, 260], [0, 10, 140, 270], [0]),
    ([0, 130, 260], [0, 2000, 400], [0, 1]),
    ([0, 100, 200, 300], [0, 100, 90, 300], [1]),
    # few queries over many keys: blocks in parts, joined
    ([0, 3, 1, 6, 9], [0, 5000, 5001, 5006, 9000], [1, 2]),
    # more sequences than a warp's lanes, bounds wrong early, late, and in several places
    (MANY[:20] + [2] + MANY[21:], ascending([9] * 44), [19, 20]),
    (MANY[:40] + [-1] + MANY[41:], ascending([40] * 44), [39, 40]),
    (MANY[:3] + [90000] + MANY[4:35] + [100] + MANY[36:], ascending([40] * 44), [2, 3, 34, 35]),
    ([0, 2] + [1] * 60 + [1, 5], ascending([300] * 63), None),
    # a thousand sequences and more
    (CROWD[:700] + [10] + CROWD[701:], ascending([1] * 1044), None),
    (CROWD[:1000] + [-1] + CROWD[1001:], ascending([1] * 1044), None),
    (THRONG[:100] + [1050] + THRONG[101:], ascending([1] * 1060), None),
    (THRONG[:1055] + [700] + THRONG[1056:], ascending([1] * 1060), None),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_prompt_sequences_that_fit_are_computed(gk, case, d, dtype):
    cq, ck, left = CASES[case]
    n_q, n_k = 1100, max(1600, max(x for x in ck if x < 100000 and x != 2000))
    good = computed(cq, ck, n_q, n_k)
    if left is not None:
        assert [i for i in range(len(cq) - 1) if i not in good] == left
    g = torch.Generator().manual_seed(case)
    q, k, v = (torch.randn(n, h, d, generator=g).to(dtype) for n, h in ((n_q, 8), (n_k, 2), (n_k, 2)))
    out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    op = gk.PromptAttention(G=2, Hq=8, d=d, dtype=dtype)
    op(q.cuda(), k.cuda(), v.cuda(), torch.tensor(cq, **I32), torch.tensor(ck, **I32), out=out, lse=lse, return_lse=True)
    with pytest.raises(gk.GraceKVError) as e:
        op.status()
    assert e.value.status == gk.GKV_EINVAL
    got, glse = out.double().cpu(), lse.double().cpu()
    rows = torch.zeros(n_q, dtype=torch.bool)
    for i in good:
        a, b = cq[i], cq[i + 1]
        want, wlse, tol, ltol = (t[a:b] for t in R.prompt(q, k, v, [a, b], [ck[i], ck[i + 1]], bf16=dtype == BF))
        assert not rows[a:b].any()
        rows[a:b] = True
        empty = torch.isinf(wlse)
        assert (got[a:b][empty] == 0).all() and torch.equal(glse[a:b][empty], wlse[empty]), i
        assert ((got[a:b] - want).abs() <= tol)[~empty].all(), i
        assert ((glse[a:b] - wlse).abs() <= ltol)[~empty].all(), i
    assert (got[~rows] == 7.0).all() and (glse[~rows] == 7.0).all()
    # the object works on
    c = torch.tensor([0, 40], **I32)
    fresh = gk.PromptAttention(G=2, Hq=8, d=d, dtype=dtype)
    args = (q[:40].cuda(), k[:40].cuda(), v[:40].cuda(), c)
    assert torch.equal(op(*args), fresh(*args))
    op.status()
