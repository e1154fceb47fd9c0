"""The bindings of the attention over caches in 16, 8 and 4 bits, without a device: host tensors, and a library that takes
down which calls are made."""
import pytest
import torch

from paper_2609_27373_gb300 import serve, wise


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 64 if name.endswith("workspace") or name.endswith("bytes") else 0
        return call


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(wise, "load", lambda: lib)
    monkeypatch.setattr(wise, "_check", lambda *a: None)
    monkeypatch.setattr(wise, "_current_raw", lambda index: 0)
    monkeypatch.setattr(wise, "_current_device", lambda: -1)  # the index of host tensors
    return lib


def make(bits):
    lists = [torch.zeros((2, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)]
    if bits == 16:
        return serve.PagedCache.over(torch.zeros((2, 3, 2, 16, 64), dtype=torch.bfloat16), *lists)
    return serve.PagedCache.over(torch.zeros((1, 3, 2, 64), dtype=torch.uint8), *lists, bits=bits, page=16, head_dim=64,
                                 dtype=torch.bfloat16)


def queries(batch=2, heads=4, q_len=3, dim=64):
    return torch.zeros((batch, heads, q_len, dim), dtype=torch.bfloat16)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_queries_of_another_shape_than_the_one_given_are_refused(lib, bits):
    """The kernel goes by `shape`: fewer rows in Q or O would be read and written past their end."""
    cache, attn = make(bits), wise.wise_prefix_attn if bits == 16 else wise.wise_kvq_attn
    Q, shape = queries(), wise.prefix_shape(make(bits), queries(), 0)
    slots = torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(64, dtype=torch.uint8)
    attn(cache, 0, Q, torch.empty_like(Q), slots, workspace=ws, shape=shape)
    attn(cache, 0, Q, torch.empty_like(Q), slots, workspace=ws)
    lib.calls.clear()
    for other in (queries(q_len=1), queries(heads=2), queries(batch=1), queries(dim=128), queries(q_len=4)):
        for q, o in ((other, torch.empty_like(other)), (Q, other), (other, Q)):
            with pytest.raises(ValueError):
                attn(cache, 0, q, o, slots, workspace=ws, shape=shape)
    for bad in (None, Q[0], Q.float()):
        with pytest.raises(ValueError):
            attn(cache, 0, bad, Q, slots, workspace=ws)
    with pytest.raises(ValueError, match="prefix_lens"):
        attn(cache, 0, Q, torch.empty_like(Q), slots, group_start=slots, workspace=ws)
    assert lib.calls == []


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_tensors_of_another_device_than_the_current_one_are_refused(lib, monkeypatch, bits):
    """Workspaces are of the current device's number of SMs, so they too are asked for on the tensors' own device."""
    cache, Q, lists = make(bits), queries(), torch.zeros(2, dtype=torch.int32)
    KV, shape = queries(heads=2), wise.prefix_shape(cache, Q, 0)
    workspace = wise.wise_prefix_attn_workspace if bits == 16 else wise.wise_kvq_attn_workspace
    calls = [lambda: cache.attend(0, Q, torch.empty_like(Q), lists), lambda: cache.write(0, lists, None, KV, KV),
             lambda: cache.read(0, KV, KV.clone(), lists), lambda: workspace(cache, shape)]
    monkeypatch.setattr(serve.PagedCache, "_use", lambda self, stream: wise._raw_stream(stream, self.index))
    monkeypatch.setattr(serve, "_empty", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
    for call in calls:
        call()
    monkeypatch.setattr(wise, "_current_device", lambda: 1)
    lib.calls.clear()
    for call in calls:
        with pytest.raises(ValueError, match="device"):
            call()
    assert lib.calls == []
