"""The host side of the quantised cache, of reads and unloads and of the attention over
shared prefixes without a GPU, with the stand-ins of test_serving_host.py."""
import types

import pytest
import torch

from paper_2608_07001_gb300 import gracekv as gk

from .test_serving_host import BF, Tensor, on_device_1, packed, pages, same, state  # noqa: F401

I32, U8 = dict(dtype=torch.int32), dict(dtype=torch.uint8)


@pytest.fixture
def calls(on_device_1):  # noqa: F811
    _, lib, now = on_device_1
    e4 = dict(dtype=torch.float8_e4m3fn)

    def make(B, quant):
        kind, sc = (e4, dict(k_scale=Tensor(4, 16, **U8), v_scale=Tensor(4, 16, **U8))) if quant else (dict(dtype=BF), {})
        return gk.PagedCache(Tensor(4, 16, 64, **kind), Tensor(4, 16, 64, **kind), Tensor(1, B, 2, 2, **I32),
                             Tensor(1, B, 2, **I32), Hq=4, **sc)
    c, plain, x = make(3, True), make(3, False), make(2, True)
    f = gk.SharedAttention(plain, x)
    q, k = Tensor(3, 4, 64), Tensor(3, 2, 64)
    made = {
        "quant_load": lambda **kw: c.load_packed(0, Tensor(5, 64), Tensor(5, 64), None, Tensor(3, dtype=torch.int64), **kw),
        "quant_append": lambda **kw: c.append(0, k, k, Tensor(3, **I32), q=q, **kw),
        "quant_attention": lambda **kw: c.attention(0, q, **kw),
        "paged_advance": lambda **kw: c.advance_by(Tensor(4, **I32), **kw),
        "paged_read": lambda **kw: c.read(0, 3, Tensor(4, **I32), **kw),
        "paged_unload": lambda **kw: plain.unload_packed(1, 7, **kw),
        "shared_attention": lambda **kw: f(0, q, Tensor(3, **I32), **kw),
        "shared_status": lambda **kw: f.status(**kw),
    }
    return made, lib, now, f


NAMES = ["quant_load", "quant_append", "quant_attention", "paged_advance", "paged_read", "paged_unload", "shared_attention", "shared_status"]


@pytest.mark.parametrize("name", NAMES)
def test_calls_are_made_on_the_tensors_device(calls, name):
    made, lib, now, _ = calls
    made[name]()
    assert lib.seen == [("gracekv_" + name, 1)] and now["device"] == 0


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device_is_refused(calls, name):
    made, lib, _, _ = calls
    with pytest.raises(gk.GraceKVError) as e:
        made[name](stream=types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=7))
    assert e.value.status == gk.GKV_EINVAL and not lib.seen


def test_caches_of_two_devices_are_refused(calls):
    _, _, _, f = calls
    f.prefix._device = torch.device("cuda", 0)
    with pytest.raises(gk.GraceKVError):
        gk.SharedAttention(f.cache, f.prefix)


def test_quantised_pages_that_the_cache_hands_out(pages):  # noqa: F811
    c = pages(quantised=True)
    assert c.K.dtype is torch.float8_e4m3fn and c.dtype is BF and c.k_scale.shape == (40, 16)
    assert {t.data_ptr() for t in c._made} >= {t.data_ptr() for t in (c.K, c.V, c.k_scale, c.v_scale, c.log_m, c.table, c.lens)}
    c.load(1, *packed([16, 17, 1, 3]))
    before = state(c)
    for bad in (packed([20, 1, 1, 1], dtype=torch.float32), packed([20, 1, 1, 1], d=128)):
        with pytest.raises((gk.GraceKVError, ValueError)):
            c.load(1, *bad)
        assert same(state(c), before)
    out = c.unload(1)
    assert out.K.shape == (37, 64) and out.K.dtype is BF and out.pos is None and out.offsets.shape == (5,)
    assert same(state(c), before)
    c.release(1)
    assert c._n_free == 40 and c.unload(1).K.shape == (0, 64)
    for b in (-1, 3):
        with pytest.raises(gk.GraceKVError):
            c.unload(b)


def test_unloads_into_given_tensors(pages):  # noqa: F811
    c = pages()
    good = [torch.zeros(9, 64, dtype=BF), torch.zeros(9, 64, dtype=BF), torch.zeros(9), torch.zeros(5, dtype=torch.int64)]
    assert c.unload_packed(0, 9, good) is good
    for i, t in ((0, torch.zeros(8, 64, dtype=BF)), (1, torch.zeros(9, 64)), (2, torch.zeros(9).double()), (3, torch.zeros(4, dtype=torch.int64)),
                 (0, torch.zeros(9 * 64 + 1, dtype=BF)[1:].view(9, 64)), (1, torch.zeros(64, 9, dtype=BF).t())):
        with pytest.raises((gk.GraceKVError, ValueError)):
            c.unload_packed(0, 9, good[:i] + [t] + good[i + 1:])
    for b, n in ((3, 9), (-1, 9), (0, -1), (0, 1 << 31)):
        with pytest.raises(gk.GraceKVError):
            c.unload_packed(b, n)


def test_a_cache_whose_pages_are_the_callers_has_no_unload():
    c = object.__new__(gk.PagedCache)
    c._free = None
    with pytest.raises(gk.GraceKVError):
        c.unload(0)
