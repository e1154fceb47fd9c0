"""PagedCache's handling of its memory, without a device: host tensors, and a library that only says how large its
workspaces are and takes down what it is called with."""
import pytest
import torch

from paper_2609_27373_gb300 import serve, wise


class Stream:
    def __init__(self, raw):
        self.cuda_stream, self.device_index = raw, -1   # -1: the index of host tensors


class Library:
    """Workspaces: 64 bytes a list entry, 1024 a request."""

    def __init__(self):
        self.workspaces = []

    def wise_kv_workspace(self, cache, n):
        return 64 * (n + 1)

    def wise_prefix_attn_workspace(self, cache, shape):
        return 1024 * shape._obj.batch

    def wise_kv_extend(self, cache, slots, n_new, n, granted, workspace, stream):
        self.workspaces.append(workspace)
        return 0

    def wise_kv_compact(self, cache, remap, n_live, workspace, stream):
        self.workspaces.append(workspace)
        return 0

    def wise_prefix_attn(self, cache, layer, shape, Q, slots, n_new, start, lens, O, workspace, ws_bytes, stream):
        assert ws_bytes >= 1024 * shape._obj.batch
        self.workspaces.append(workspace)
        return 0

    def wise_kv_fork(self, *args):
        return 0

    wise_kv_write = wise_kv_drop = wise_kv_fork


class Torch:
    """What stands in for torch's streams: the current one, and which tensors were recorded on which."""

    def __init__(self):
        self.current, self.recorded = Stream(0), []


@pytest.fixture
def host(monkeypatch):
    t = Torch()
    t.lib = Library()
    monkeypatch.setattr(wise, "load", lambda: t.lib)
    monkeypatch.setattr(wise, "_check", lambda *a: None)
    monkeypatch.setattr(wise, "_current_raw", lambda index: t.current.cuda_stream)
    monkeypatch.setattr(wise, "_current_device", lambda: -1)
    monkeypatch.setattr(serve, "_empty", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: t.current)
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda x, s: t.recorded.append((x.data_ptr(), s.cuda_stream)), raising=False)
    return t


def make():
    return serve.PagedCache.over(torch.zeros((2, 8, 2, 16, 64), dtype=torch.bfloat16),
                                 torch.zeros((600, 4), dtype=torch.int32), torch.zeros(600, dtype=torch.int32),
                                 torch.zeros(8, dtype=torch.int32))


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


def attend(cache, batch, stream=None):
    Q = torch.zeros((batch, 4, 1, 64), dtype=torch.bfloat16)
    cache.attend(0, Q, torch.empty_like(Q), i32(batch), stream=stream)


def everything(cache, stream=None):
    K = torch.zeros((2, 2, 1, 64), dtype=torch.bfloat16)
    return [lambda: cache.fork(i32(2), i32(2), stream=stream), lambda: cache.extend(i32(2), i32(2), stream=stream),
            lambda: cache.write(0, i32(2), None, K, K, stream=stream), lambda: cache.drop(i32(2), i32(2), stream=stream),
            lambda: cache.compact(stream=stream), lambda: attend(cache, 2, stream)]


@pytest.mark.parametrize("given", [True, False])
def test_every_stream_that_uses_the_cache_is_recorded_on_its_memory(host, given):
    """The pool, the lists and the workspaces must not be handed out again while a stream that they do not come from
    still reads them."""
    for k in range(len(everything(make()))):
        cache, side = make(), Stream(77)
        host.recorded.clear()
        host.current = Stream(0) if given else side
        everything(cache, side if given else None)[k]()
        own = {t.data_ptr() for t in (cache.pool, cache.table, cache.lens, cache.refs)}
        assert {p for p, s in host.recorded if s == 77} >= own, k


def test_workspaces_are_recorded_on_streams_that_came_before_and_after_them(host):
    cache, a, b = make(), Stream(5), Stream(6)
    cache.fork(i32(1), i32(1), stream=a)
    attend(cache, 1, a)
    first = host.lib.workspaces[-1]
    cache.extend(i32(1), i32(1), stream=b)
    attend(cache, 1, b)
    assert host.lib.workspaces[-1] == first
    for ws in host.lib.workspaces:
        assert {(ws, 5), (ws, 6)} <= set(host.recorded)
    n = len(host.recorded)
    attend(cache, 1, a)
    attend(cache, 1, b)
    assert len(host.recorded) == n   # once a stream


def extend(cache, n):
    cache.extend(i32(n), i32(n))


def test_a_workspace_that_a_graph_may_hold_is_kept(host):
    """A graph that was captured with a small batch still writes to the workspace of that time when larger batches
    and longer lists have come since."""
    cache = make()
    attend(cache, 2)
    extend(cache, 2)
    small = list(host.lib.workspaces)
    for n in (3, 9, 40, 41, 500):
        attend(cache, n)
        extend(cache, n)
    held = {ws.data_ptr(): ws.numel() for ws in cache._workspaces}
    assert set(host.lib.workspaces) <= set(held) and set(small) <= set(held)
    assert len(set(host.lib.workspaces)) == len(held) >= 6
    # What is kept beside the two in use is no more than those.
    assert sum(held.values()) <= 2 * (cache._attn_ws.numel() + cache._kv_ws.numel())
    attend(cache, 2)
    extend(cache, 2)
    assert host.lib.workspaces[-2:] == [cache._attn_ws.data_ptr(), cache._kv_ws.data_ptr()]


def verify(stream=None):
    p = torch.zeros((2, 2, 10))
    return wise.wise_verify_draft(p, p[:, :1].contiguous(), i32((2, 1)), None, torch.zeros((2, 1)), torch.zeros(2),
                                  i32(2), i32((2, 2)), stream)


def test_tensors_of_another_device_than_the_current_one_are_refused(host, monkeypatch):
    """The library takes the current device's status word, its number of SMs and its streams: nothing is launched
    for tensors that lie elsewhere."""
    cache = make()
    shape = wise.prefix_shape(cache, torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16), 0)
    calls = everything(cache) + [lambda: wise.wise_prefix_attn_workspace(cache, shape)]
    for call in calls:
        call()
    monkeypatch.setattr(wise, "_current_device", lambda: 1)
    monkeypatch.setattr(wise, "load", lambda: pytest.fail("the library was called"))
    fresh = make()
    for call in everything(cache) + everything(fresh) + [lambda: wise.wise_prefix_attn_workspace(cache, shape)]:
        with pytest.raises(ValueError, match="device"):
            call()


def test_a_stream_of_another_device_is_refused(host, monkeypatch):
    cache, far = make(), Stream(9)
    far.device_index = 1
    monkeypatch.setattr(wise, "load", lambda: pytest.fail("the library was called"))
    for call in everything(cache, far):
        with pytest.raises(ValueError, match="stream"):
            call()


def test_the_binding_of_the_verification_looks_at_the_device(host, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    host.lib.wise_verify_draft = lambda *a: 0
    verify()
    far = Stream(9)
    far.device_index = 1
    with pytest.raises(ValueError, match="stream"):
        verify(far)
    monkeypatch.setattr(wise, "_current_device", lambda: 1)
    host.lib.wise_verify_draft = lambda *a: pytest.fail("the library was called")
    with pytest.raises(ValueError, match="device"):
        verify()
