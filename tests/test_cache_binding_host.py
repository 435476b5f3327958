"""The binding of the rotation and the paged cache, on the CPU: what it hands to the library and what it refuses.  The library's calls are recorded, none is made."""
import ctypes as C

import pytest


class Calls:
    """In the library's place: the arguments of every call."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        return lambda *args: (self.made.append((name, args)), 0)[1]


class OnDevice:
    """A tensor that says it lies on device 1."""

    def __init__(self, t):
        self.t, self.shape, self.dtype, self.device = t, t.shape, t.dtype, "cuda:1"

    def get_device(self):
        return 1

    def stride(self, *dim):
        return self.t.stride(*dim)

    def data_ptr(self):
        return 0x10000


@pytest.fixture
def calls(lib, monkeypatch):
    """The current device is "the CPU" (-1), where tensors are made; nothing is called."""
    import torch
    made = Calls()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(lib, "_current", lambda stream: (None, -1))
    monkeypatch.setattr(lib, "_lib", made)
    return made


def _cache(lib):
    import torch
    pages = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    return lib.paged_cache(pages, torch.zeros_like(pages), torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32))


def test_handles_of_another_device_are_refused(lib, calls, monkeypatch):
    """A rotation and a cache made on one device, used with another one current and every tensor of the call there."""
    import torch
    r, cache = lib.rope(torch.zeros(1, 1, 1, dtype=torch.int32), torch.zeros(32)), _cache(lib)
    x, o = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 2, 64)
    shp = lib.shape(1, 2, 2, 64, 1, 16, 1.0)
    use = {"rope": lambda x, o: lib.burst_attn_rope(shp, r, x, o),
           "append": lambda x, o: lib.burst_attn_cache_append(shp, cache, x, x),
           "append, rotation": lambda x, o: lib.burst_attn_cache_append(shp, elsewhere, x, x, rope=r, q=x, q_out=x),
           "decode": lambda x, o: lib.burst_attn_decode(shp, cache, x, o)}
    elsewhere = cache
    for call in use.values():
        call(x, o)                                                         # on their own device they are taken
    assert len(calls.made) == 4
    monkeypatch.setattr(lib, "_current", lambda stream: (None, 1))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    elsewhere = _cache_on_device_1(lib)
    for name, call in use.items():
        with pytest.raises(ValueError, match="current device"):
            call(OnDevice(x), OnDevice(o))
    assert len(calls.made) == 4
    lib.burst_attn_cache_append(shp, elsewhere, OnDevice(x), OnDevice(x))  # (all of it on device 1)
    assert len(calls.made) == 5


def _cache_on_device_1(lib):
    import torch
    pages = OnDevice(torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16))
    pages.dim, pages.size = pages.t.dim, pages.t.size
    numbers = []
    for t in (torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32)):
        x = OnDevice(t)
        x.dim, x.size, x.numel = t.dim, t.size, t.numel
        numbers.append(x)
    return lib.paged_cache(pages, pages, *numbers)


def test_a_table_of_one_sequence_has_any_stride(lib, monkeypatch):
    """A dimension of one entry: whatever its stride is (1 here, as a column of a larger table turned round), no row of the table is skipped."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    pages = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    table = torch.zeros(5, 1, dtype=torch.int32).t()
    assert table.shape == (1, 5) and table.stride() == (1, 1)
    cache = lib.paged_cache(pages, torch.zeros_like(pages), table, torch.zeros(1, dtype=torch.int32))
    assert lib.burst_attn_decode_plan(lib.shape(1, 2, 2, 64, 1, 80, 1.0), cache)[2]
    two = torch.zeros(2, 9, dtype=torch.int32)[:, :5]
    assert lib.paged_cache(pages, torch.zeros_like(pages), two, torch.zeros(2, dtype=torch.int32)).table_stride == 9
