"""Rotation and append of a chunk without rows, on the CPU: nothing is launched, and tensors without rows need no memory (an empty torch tensor has none)."""
import pytest

from tests.test_cache_abi_host import Calls


@pytest.fixture
def calls(lib):
    return Calls(lib)


def test_calls_without_rows(lib, calls):
    c, none = calls, calls.tensor(0)
    shape = c.shape(sq=0)
    assert c.turn(shape=shape) == lib.BURST_OK and c.append(shape=shape) == lib.BURST_OK                  # with memory
    no_places = c.changed(c.rope, positions=None)
    assert c.turn(shape=shape, rope=no_places, q=none, q_out=none, k=none, k_out=none) == lib.BURST_OK
    assert c.turn(shape=shape, rope=no_places, q=none, q_out=c.tensor(0, dtype=1), k=None, k_out=None) == lib.BURST_OK
    assert c.append(shape=shape, k=none, v=none, rope=no_places, q=none, q_out=none) == lib.BURST_OK
    assert c.append(shape=shape, k=none, v=none, rope=None, q=None, q_out=None, new=None) == lib.BURST_OK


def test_what_is_wrong_without_rows_too(lib, calls):
    """Everything else is checked as with rows."""
    INV, UNS, c, none = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, calls, calls.tensor(0)
    shape = c.shape(sq=0)
    assert c.turn(shape=shape, q=None) == INV and c.turn(shape=shape, k=None) == INV and c.append(shape=shape, v=None) == INV
    assert c.turn(shape=shape, q=c.tensor(0, dtype=2)) == INV and c.append(shape=shape, k=c.tensor(0, dtype=1)) == UNS
    assert c.turn(shape=shape, rope=c.changed(c.rope, inv_freq=None)) == INV
    assert c.turn(shape=shape, rope=c.changed(c.rope, positions=0x2001)) == INV
    assert c.append(shape=shape, cache=c.changed(c.cache, rows=None)) == INV
    for call in (c.turn, c.append):                                       # with rows there is no tensor without memory
        assert call(q=none) == INV and call(q_out=none) == INV and call(k=none) == INV
        assert call(rope=c.changed(c.rope, positions=None)) == INV
    assert c.turn(k_out=none) == INV and c.append(v=none) == INV


def test_empty_tensors_through_the_binding(lib, monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)          # as if the CPU were the current device: no launch, no GPU
    monkeypatch.setattr(lib, "_current", lambda stream: (None, -1))
    x = torch.zeros(2, 0, 2, 64, dtype=torch.bfloat16)
    y, k = torch.zeros(2, 0, 2, 64), torch.zeros(2, 5, 1, 64, dtype=torch.bfloat16)[:, 5:]
    r = lib.rope(torch.zeros(1, 2, 0, dtype=torch.int32), torch.ones(32))
    shp = lib.shape(2, 2, 1, 64, 0, 0, 1.0)
    lib.burst_attn_rope(shp, r, x, x)
    lib.burst_attn_rope(shp, r, x, y, k, torch.empty_like(k))
    pages = torch.ones(3, 16, 1, 64, dtype=torch.bfloat16)
    cache = lib.paged_cache(pages, pages.clone(), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    lib.burst_attn_cache_append(shp, cache, k, k, rope=r, q=x, q_out=torch.empty_like(x), new_rows=torch.zeros(2, dtype=torch.int32))
    assert (pages == 1).all()
