"""A cache made on a device that is not the current one: the library, which refuses calls from another current device, is called with
the cache's device current.  CPU only: torch's CUDA calls and the library's are fakes."""
import contextlib

import pytest
import torch

from paper_2607_09385_b200 import binding as B
from paper_2607_09385_b200 import cache as C


@pytest.fixture
def fake(monkeypatch):
    """Two devices, device 0 current; the library notes which one is current in each call."""
    calls, current = [], [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d).index
        yield
        current[0] = before

    def called(name):
        def call(*args):
            calls.append((name, current[0]))
            return B.STEEL_OK if name == "create" or current[0] == 1 else B.STEEL_ERR_INVALID_ARG
        return call

    class Library:
        steel_cache_reset = staticmethod(called("reset"))

    on_cpu = lambda f: lambda *a, device=None, **kw: f(*a, **kw)  # noqa: E731
    for name in ("empty", "zeros"):
        monkeypatch.setattr(torch, name, on_cpu(getattr(torch, name)))
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    sizes = C.steel_cache_sizes(C.CacheParams(1, 4, 16, 1, 64, 2, 2))
    monkeypatch.setattr(C, "steel_cache_sizes", lambda params: sizes)
    monkeypatch.setattr(C, "steel_cache_create", lambda params, memory: called("create")() and None)  # no handle to destroy
    monkeypatch.setattr(C, "load_library", lambda: Library)
    monkeypatch.setattr(B, "_stream_getter", lambda: lambda index: 0)
    return calls


@pytest.mark.parametrize("device", ["cuda:1", torch.device("cuda", 1)])
def test_a_cache_on_another_device(fake, device):
    cache = C.SteelCache(1, 4, 16, 1, 64, 2, 2, device=device)
    assert cache.device_index == 1 and fake == [("create", 1), ("reset", 1)]
    cache.close()


def test_a_cache_needs_a_cuda_device(fake):
    with pytest.raises(AssertionError):
        C.SteelCache(1, 4, 16, 1, 64, 2, 2, device="cpu")
    assert fake == []
