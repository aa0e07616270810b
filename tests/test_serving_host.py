"""The host side of the serving objects without a GPU: tensors and the C library
are stand-ins, so that what reaches a launch, and what does not, can be seen."""
import contextlib
import types
from ctypes import c_int32

import pytest
import torch

from paper_2608_07001_gb300 import gracekv as gk

BF = torch.bfloat16


class Tensor:
    """A CUDA tensor as the wrappers look at it."""
    is_cuda = True

    def __init__(self, *shape, dtype=BF, device="cuda:1"):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device(device)

    def dim(self):
        return len(self.shape)

    def stride(self):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s)

    def data_ptr(self):
        return 1 << 20

    def is_contiguous(self):
        return True

    def record_stream(self, stream):
        pass


class Lib:
    """Every call succeeds and notes the device that was current."""

    def __init__(self, now):
        self.now, self.seen = now, []

    def __getattr__(self, name):
        def call(*args):
            if not name.endswith("workspace_size"):
                self.seen.append((name, self.now["device"]))
            return gk.GKV_OK
        return call


@pytest.fixture
def on_device_1(monkeypatch):
    """Objects whose tensors are on cuda:1 while cuda:0 is current: (their calls, the library)."""
    now = {"device": 0}
    lib = Lib(now)

    @contextlib.contextmanager
    def device(d):
        before, now["device"] = now["device"], torch.device(d).index
        try:
            yield
        finally:
            now["device"] = before

    def make_workspace(self, n, dev):
        self.workspace, self._device, self._ws, self._own_stream = Tensor(n, dtype=torch.uint8), torch.device("cuda", 1), 1 << 20, 0
        self._made, self._used_on = [self.workspace], set()

    monkeypatch.setattr(gk, "lib", lambda: lib)
    monkeypatch.setattr(gk._Workspace, "_make_workspace", make_workspace)
    monkeypatch.setattr(gk, "_empty_like_on", lambda stream, shape, dtype, dev: Tensor(*shape, dtype=dtype, device=dev))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now["device"], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 0, raising=False)
    i32 = dict(dtype=torch.int32)
    p = gk.PromptAttention(G=2, Hq=4, d=64, dtype=BF, device="cuda:1")
    c = gk.PagedCache(Tensor(4, 16, 64), Tensor(4, 16, 64), Tensor(1, 3, 2, 2, **i32), Tensor(1, 3, 2, **i32), Hq=4)
    q, k, cu = Tensor(3, 4, 64), Tensor(3, 2, 64), Tensor(4, **i32)
    calls = {
        "prompt_attention": lambda **kw: p(q, k, k, cu, **kw), "prompt_status": lambda **kw: p.status(**kw),
        "paged_load": lambda **kw: c.load_packed(0, Tensor(5, 64), Tensor(5, 64), None, Tensor(3, dtype=torch.int64), **kw),
        "paged_advance": lambda **kw: c.advance_by(cu, **kw), "paged_append": lambda **kw: c.append(0, k, k, Tensor(3, **i32), q=q, **kw),
        "paged_attention": lambda **kw: c.attention(0, q, **kw), "paged_status": lambda **kw: c.status(**kw),
    }
    return calls, lib, now


NAMES = ["prompt_attention", "prompt_status", "paged_load", "paged_advance", "paged_append", "paged_attention", "paged_status"]


@pytest.mark.parametrize("name", NAMES)
def test_calls_are_made_on_the_tensors_device(on_device_1, name):
    # the library launches on the current device; the raw stream of another one's default is 0 there too
    calls, lib, now = on_device_1
    calls[name]()
    assert lib.seen == [("gracekv_" + name, 1)] and now["device"] == 0
    now["device"] = 1
    calls[name]()
    assert lib.seen[1:] == [("gracekv_" + name, 1)] and now["device"] == 1


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device_is_refused(on_device_1, name):
    calls, lib, _ = on_device_1
    stream = types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=7)
    with pytest.raises(gk.GraceKVError) as e:
        calls[name](stream=stream)
    assert e.value.status == gk.GKV_EINVAL and not lib.seen
    calls[name](stream=types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=7))
    assert lib.seen == [("gracekv_" + name, 1)]


# ------------------------------------------------------- pages that the cache hands out
L, B, G, HQ, D, PS = 2, 3, 2, 4, 64, 16


class PageLib:
    """gracekv_paged_advance on host memory; the other calls succeed without doing anything."""

    def __init__(self):
        self.cache = None

    def gracekv_paged_advance(self, ref, cu, stream):
        c = self.cache
        n = torch.tensor((c_int32 * (c.B + 1)).from_address(cu)).diff() if cu else None
        for b in range(c.B):
            c.lens[:, b] += (c.lens[:, b] > 0).int() if n is None else int(n[b])
        return gk.GKV_OK

    def __getattr__(self, name):
        return lambda *a: gk.GKV_OK


@pytest.fixture
def pages(monkeypatch):
    """A function that makes caches of their own pages on the CPU."""
    lib = PageLib()

    def make_workspace(self, n, dev):
        self.workspace, self._device, self._ws, self._own_stream = torch.zeros(256, dtype=torch.uint8), torch.device("cpu"), 0, 0
        self._made, self._used_on = [self.workspace], set()

    monkeypatch.setattr(gk, "lib", lambda: lib)
    monkeypatch.setattr(gk._Workspace, "_make_workspace", make_workspace)
    monkeypatch.setattr(gk._Workspace, "_on", lambda self, stream, *t: 0)
    monkeypatch.setattr(gk._Workspace, "_run", lambda self, call, *a: gk._raise(call(*a)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())

    def make(**kw):
        lib.cache = gk.PagedCache.allocate(**(dict(L=L, B=B, G=G, Hq=HQ, d=D, dtype=BF, n_pages=40, max_pages=5, page_size=PS,
                                                   device="cpu") | kw))
        return lib.cache
    return make


def packed(counts, d=D, dtype=BF, lg=None):
    off = torch.tensor([0] + list(counts)).cumsum(0)
    c = gk.Cache.empty(int(off[-1]), d, len(counts) if lg is None else lg, dtype, device="cpu")
    c.log_m.zero_()
    c.offsets.copy_(off) if lg is None else c.offsets.zero_()
    return c, int(off[-1])


def state(c):
    return c.table.clone(), c.lens.clone(), c._host_lens.copy(), c._host_table.copy(), c._n_free, sorted(c._free[:c._n_free])


def same(a, b):
    return all(torch.equal(x, y) if isinstance(x, torch.Tensor) else (x == y) if isinstance(x, (int, list)) else (x == y).all()
               for x, y in zip(a, b))


def test_a_refused_load_changes_nothing(pages):
    c = pages()
    c.load(1, *packed([16, 17, 1, 3]))
    before = state(c)
    good, n = packed([20, 1, 1, 1])
    bad = [
        (1, packed([20, 1, 1, 1], dtype=torch.float32)[0], n),            # another type
        (1, packed([20, 1, 1, 1], d=128)[0], n),                          # another head size
        (1, packed([20, 1, 1, 1], lg=6)[0], n),                           # offsets of another L x G
        (1, good, n + 1), (1, good, -1), (3, good, n), (-1, good, n),
        (1, gk.Cache(*(getattr(good, f) if f != "V" else good.V[:5] for f in ("K", "V", "pos", "log_m", "src_lo", "src_hi", "offsets"))), n),
        (1, gk.Cache(*(getattr(good, f) if f != "log_m" else good.log_m.double() for f in ("K", "V", "pos", "log_m", "src_lo", "src_hi", "offsets"))), n),
        (1, packed([90, 1, 1, 1])[0], 93),                                # more pages than a sequence may have
    ]
    for b, cache, m in bad:
        with pytest.raises((gk.GraceKVError, ValueError)):
            c.load(b, cache, m)
        assert same(state(c), before), (b, m)
    with pytest.MonkeyPatch.context() as m:                               # a stream of another device
        def refuse(self, stream, *t):
            raise gk.GraceKVError(gk.GKV_EINVAL, "stream")
        m.setattr(gk._Workspace, "_on", refuse)
        with pytest.raises(gk.GraceKVError):
            c.load(1, good, n, stream=object())
        assert same(state(c), before)
    c.load(1, good, n)
    assert c._host_lens[:, 1].tolist() == [[20, 1], [1, 1]] and c._host_lens[:, [0, 2]].sum() == 0


def test_a_request_that_takes_a_token_takes_it_in_every_head(pages):
    # a head that holds nothing belongs to its request all the same; a request without entries is idle
    c = pages()
    c.load(1, *packed([16, 0, 0, 3]))
    c.lens[:, 1] = torch.tensor([[16, 0], [0, 3]], dtype=torch.int32)         # as gracekv_paged_load writes them
    for step in range(1, 4):
        assert c.advance() is None
        want = torch.zeros(L, B, G, dtype=torch.int32)
        want[:, 1] = torch.tensor([[16, 0], [0, 3]]) + step
        assert torch.equal(c.lens, want) and (c._host_lens == want.numpy()).all()
        need = -(-want // PS)
        assert torch.equal((c.table >= 0).sum(-1), need)                      # every entry has its page
    c.release(1)
    c.lens[:, 1] = 0
    assert c.advance() is None and int(c.lens.sum()) == 0 and c._n_free == 40


def test_multiplicities_are_not_dropped(pages):
    # a cache without log m takes a packed one whose entries are single tokens, and no other
    c = pages(log_m=False)
    cache, n = packed([16, 17, 1, 3])
    c.load(1, cache, n)
    before = state(c)
    cache.log_m[20] = 0.7
    with pytest.raises(gk.GraceKVError) as e:
        c.load(1, cache, n)
    assert e.value.status == gk.GKV_EINVAL and same(state(c), before)
    cache.log_m[20] = 0.0
    more = gk.Cache.empty(n + 5, D, L * G, BF, device="cpu")        # capacity past the entries holds anything
    more.log_m.fill_(3.0)
    more.log_m[:n] = 0
    more.offsets.copy_(cache.offsets)
    c.load(1, more, n)


def test_a_released_slot_leads_to_no_page(pages):
    # words of a page that has gone back must not be followed: the page is another request's next
    c = pages()
    c.load(1, *packed([40, 17, 1, 3]))
    c.load(2, *packed([5, 5, 5, 5]))
    kept = c.table[:, 2].clone()
    c.release(1)
    assert (c.table[:, 1] == -1).all() and torch.equal(c.table[:, 2], kept)
    c.load(1, *packed([1, 1, 1, 1]))
    assert torch.equal((c.table >= 0).sum(-1)[:, 1], torch.ones(L, G, dtype=torch.int64))
    assert (torch.from_numpy(c._host_table) == c.table).all()


def test_what_an_object_made_stays_for_the_streams_it_is_used_on(pages, monkeypatch):
    # the workspace, and the pool, table and lengths of a cache of its own pages: none of them is reused while work of
    # another current stream is queued
    monkeypatch.undo()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(
        synchronize=lambda: None, cuda_stream=0, device=torch.device("cpu")))
    seen = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: seen.append(self.data_ptr()))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: now[0], raising=False)
    now = [0]
    c = gk.PagedCache.allocate(L=L, B=B, G=G, Hq=HQ, d=D, dtype=BF, n_pages=4, max_pages=2, page_size=PS, device="cpu")
    own = {t.data_ptr() for t in (c.workspace, c.K, c.V, c.log_m, c.table, c.lens)}
    assert len(own) == 6
    c._on(None)
    assert not seen                                          # the stream they were made on
    now[0] = 5
    c._on(None)
    assert set(seen) == own
    seen.clear()
    theirs = gk.PagedCache(c.K, c.V, c.table, c.lens, log_m=c.log_m, Hq=HQ)
    theirs._on(None)
    assert seen == [theirs.workspace.data_ptr()]             # the caller's tensors are the caller's to keep
