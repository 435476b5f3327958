"""Rotation, paged cache and attention of one token at the C-ABI boundary, on the CPU: struct layouts, and that every argument the
interface rules out is refused before anything could reach a GPU (the addresses are made up and never dereferenced)."""
import ctypes as C

import pytest

INF = float("inf")


def test_struct_layouts_match_the_header(lib):
    assert C.sizeof(lib.burst_rope_t) == 16 + 8 * 4 + 64
    assert lib.burst_rope_t.axis_of_pair.offset == 48
    assert C.sizeof(lib.burst_cache_t) == 2 * 40 + 8 + 8 + 8 * 5
    assert lib.burst_cache_t.table.offset == 96


class Calls:
    """The three calls on valid arguments, each of which a test replaces."""

    def __init__(self, lib):
        self.lib, self.raw = lib, lib.raw()
        self.rope = lib.burst_rope_t(3, 64, 0, 0, 0x1000, 0x2000, 4096, 512, (C.c_uint8 * 64)(*([0] * 10 + [1] * 10 + [2] * 12)))
        page = (1 << 16, 1 << 10, 128)
        self.cache = lib.burst_cache_t(lib.burst_tensor_t(0x100000, 0, 0, *page), lib.burst_tensor_t(0x900000, 0, 0, *page), 100, 64, 32,
                                       0x3000, 32, 0x4000, None, None)
        self.t = self.tensor()

    def tensor(self, ptr=0x10000, dtype=0, strides=(1 << 20, 1 << 12, 128)):
        return self.lib.burst_tensor_t(ptr, dtype, 0, *strides)

    def shape(self, batch=2, q_heads=8, kv_heads=4, head_dim=128, sq=5, sk=2048, scale=0.1):
        return self.lib.shape(batch, q_heads, kv_heads, head_dim, sq, sk, scale)

    def changed(self, struct, **kw):
        copy = type(struct).from_buffer_copy(struct)
        for name, value in kw.items():
            setattr(copy, name, value)
        return copy

    def ref(self, x):
        """Structs by reference; tensors and row vectors, which these calls take as bytes, as those."""
        return None if x is None else bytes(x) if isinstance(x, (self.lib.burst_tensor_t, self.lib.burst_rowvec_t)) else C.byref(x)

    def turn(self, **kw):
        a = dict(shape=self.shape(), rope=self.rope, q=self.t, q_out=self.tensor(0x20000), k=self.tensor(0x30000), k_out=self.tensor(0x40000))
        a.update(kw)
        return self.raw.burst_attn_rope(*[self.ref(a[n]) for n in ("shape", "rope", "q", "q_out", "k", "k_out")], 0, None)

    def append(self, **kw):
        a = dict(shape=self.shape(), cache=self.cache, k=self.t, v=self.tensor(0x20000), new=0x5000, rope=self.rope, q=self.tensor(0x30000),
                 q_out=self.tensor(0x40000))
        a.update(kw)
        return self.raw.burst_attn_cache_append(self.ref(a["shape"]), self.ref(a["cache"]), self.ref(a["k"]), self.ref(a["v"]), a["new"],
                                                self.ref(a["rope"]), self.ref(a["q"]), self.ref(a["q_out"]), None)

    def decode(self, ws=0x700000, ws_bytes=1 << 40, **kw):
        a = dict(shape=self.shape(sq=1), cache=self.cache, q=self.t, first=None, o=self.tensor(0x20000),
                 lse=self.lib.burst_rowvec_t(0x30000, 8, 1))
        a.update(kw)
        return self.raw.burst_attn_decode(self.ref(a["shape"]), self.ref(a["cache"]), self.ref(a["q"]), a["first"], self.ref(a["o"]),
                                          self.ref(a["lse"]), ws, ws_bytes, None)


@pytest.fixture
def calls(lib):
    return Calls(lib)


def test_rotation_refusals(lib, calls):
    INV, UNS, c = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, calls
    for field, value, status in (("n_axes", 0, INV), ("n_axes", 4, INV), ("n_axes", 2, INV), ("rotary_dim", 0, INV), ("rotary_dim", -16, INV),
                                 ("rotary_dim", 130, INV), ("rotary_dim", 144, INV), ("rotary_dim", 17, INV), ("rotary_dim", 8, UNS),
                                 ("rotary_dim", 40, UNS), ("inv_freq", None, INV), ("inv_freq", 0x1002, INV), ("positions", None, INV),
                                 ("positions", 0x2001, INV), ("stride_axis", -1, INV), ("stride_b", -1, INV), ("stride_b", 1 << 62, INV)):
        assert c.turn(rope=c.changed(c.rope, **{field: value})) == status, (field, value)
        assert c.append(rope=c.changed(c.rope, **{field: value})) == status, (field, value)
    assert c.turn(rope=None) == INV
    assert c.turn(shape=c.shape(head_dim=64), rope=c.changed(c.rope, rotary_dim=80)) == INV
    assert c.turn(shape=c.shape(head_dim=96)) == UNS
    assert c.turn(shape=c.shape(sq=-1)) == INV
    assert c.turn(shape=c.shape(batch=1 << 10, sq=1 << 22)) == INV        # q_out's batch stride does not cover its rows
    assert c.turn(shape=c.shape(batch=1 << 10, sq=1 << 22), q_out=c.tensor(0x20000, strides=(1 << 36, 1 << 12, 128)), k=None, k_out=None) == UNS
    assert c.turn(q=None) == INV and c.turn(q_out=None) == INV and c.turn(k=None) == INV and c.turn(k_out=None) == INV
    assert c.turn(q=c.tensor(0x10008)) == INV
    assert c.turn(q_out=c.tensor(0x20000, strides=(1 << 20, 1 << 12, 64))) == INV     # heads overlap
    assert c.turn(q_out=c.tensor(0x20000, strides=(1 << 20, 0, 128))) == INV
    assert c.turn(q=c.tensor(dtype=2)) == INV                                         # e4m3 is the cache's type alone
    assert c.turn(q=c.t, q_out=c.tensor(dtype=1)) == INV                              # in place as another type
    assert c.turn(q=c.t, q_out=c.tensor(strides=(1 << 20, 1 << 13, 128))) == INV      # ... or with other strides
    assert c.turn(k_out=c.tensor(0x20000)) == INV                                     # both results in one place


def test_append_refusals(lib, calls):
    INV, UNS, c = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, calls
    _cache_refusals(lib, c, c.append)
    assert c.append(k=None) == INV and c.append(v=None) == INV and c.append(q=None) == INV and c.append(q_out=None) == INV
    assert c.append(rope=None) == INV                                                 # queries that nothing is done to
    assert c.append(new=0x5001) == INV
    assert c.append(k=c.tensor(dtype=1)) == UNS and c.append(v=c.tensor(dtype=1)) == UNS and c.append(q=c.tensor(0x30000, dtype=1)) == UNS
    assert c.append(k=c.tensor(dtype=2)) == INV
    assert c.append(q_out=c.tensor(0x40000, strides=(0, 1 << 12, 128))) == INV
    page = (1 << 16, 1 << 10, 64)                                                     # heads overlap: read they may, written not
    same = c.changed(c.cache, k=c.tensor(0x100000, 0, page), v=c.tensor(0x900000, 0, page))
    assert c.append(cache=same) == INV
    assert c.append(cache=c.changed(c.cache, v=c.cache.k)) == INV                     # keys and values in one place


def test_decode_refusals(lib, calls):
    INV, UNS, c = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, calls
    _cache_refusals(lib, c, lambda shape=None, **kw: c.decode(shape=shape or c.shape(sq=1), **kw))
    assert c.decode(shape=c.shape(sq=2)) == INV and c.decode(shape=c.shape(sq=0)) == INV
    assert c.decode(shape=c.shape(sq=1, sk=2049)) == INV                              # 32 pages of 64 rows
    assert c.decode(shape=c.shape(sq=1, head_dim=32)) == UNS
    assert c.decode(shape=c.shape(sq=1, scale=INF)) == INV
    assert c.decode(shape=c.shape(sq=1, batch=1 << 22), o=c.tensor(0x20000, strides=(1 << 12, 1 << 12, 128))) == UNS
    assert c.decode(q=None) == INV and c.decode(o=None) == INV
    assert c.decode(q=c.tensor(dtype=1)) == UNS
    assert c.decode(o=c.tensor(0x20000, strides=(0, 1 << 12, 128))) == INV
    assert c.decode(lse=lib.burst_rowvec_t(0x30002, 8, 1)) == INV
    assert c.decode(lse=lib.burst_rowvec_t(0x30000, 4, 1)) == INV                     # 8 heads of a sequence, the next one 4 on
    assert c.decode(first=0x5003) == INV
    need = lib.burst_attn_decode_workspace_bytes(c.shape(sq=1))
    if need > 0:
        assert c.decode(ws=None) == INV and c.decode(ws=0x700010) == INV and c.decode(ws_bytes=need - 1) == INV
    raw = lib.raw()
    for bad in (c.shape(sq=2), c.shape(sq=1, q_heads=9), c.shape(sq=1, sk=-1), c.shape(sq=1, head_dim=256)):
        assert raw.burst_attn_decode_workspace_bytes(C.byref(bad)) == -1
    assert raw.burst_attn_decode_workspace_bytes(None) == -1


def _cache_refusals(lib, c, call):
    INV, UNS = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED
    for field, value, status in (("n_pages", 0, INV), ("n_pages", 1 << 31, UNS), ("page_rows", 0, INV), ("page_rows", (1 << 20) + 1, UNS),
                                 ("table_cols", 0, INV), ("table_cols", (1 << 24) + 1, UNS), ("table", None, INV), ("table", 0x3002, INV),
                                 ("table_stride", 31, INV), ("table_stride", -1, INV), ("table_stride", 1 << 60, INV), ("rows", None, INV),
                                 ("rows", 0x4001, INV), ("k_scale", 0x6000, INV), ("v_scale", 0x6000, INV)):
        assert call(cache=c.changed(c.cache, **{field: value})) == status, (field, value)
    assert call(cache=None) == INV
    page = (1 << 16, 1 << 10, 128)
    for bad, status in ((c.tensor(0, 0, page), INV), (c.tensor(0x100008, 0, page), INV), (c.tensor(0x100000, 1, page), UNS),
                        (c.tensor(0x100000, 3, page), INV), (c.tensor(0x100000, 2, page), UNS), (c.tensor(0x100000, 0, (1 << 16, 1 << 10, 136)), UNS),
                        (c.tensor(0x100000, 0, (1 << 16, 1 << 10, 132)), INV), (c.tensor(0x100000, 0, (-(1 << 16), 1 << 10, 128)), INV),
                        (c.tensor(0x100000, 0, (1 << 16, 1 << 25, 128)), UNS)):
        assert call(cache=c.changed(c.cache, k=bad)) == status
        assert call(cache=c.changed(c.cache, v=bad)) == status
    f8 = c.changed(c.cache, k=c.tensor(0x100000, 2, page), v=c.tensor(0x900000, 2, page), k_scale=0x6002)
    assert call(cache=f8) == INV
    odd = (1 << 16, 1 << 10, 136)                                                     # 8-byte steps of e4m3
    assert call(cache=c.changed(c.cache, k=c.tensor(0x100000, 2, odd), v=c.tensor(0x900000, 2, odd))) == INV
    far = (1 << 58, 1 << 10, 128)
    assert call(cache=c.changed(c.cache, k=c.tensor(0x100000, 0, far), v=c.tensor(0x900000, 0, far))) == INV
    assert call(shape=c.shape(kv_heads=3, sq=1)) == INV


def test_tensors_of_the_wrong_kind_are_refused_by_the_binding(lib, monkeypatch):
    import torch
    cpu = torch.zeros(1, 4, 2, 64)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        lib.rope(torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(ValueError, match="current device"):
        lib.paged_cache(cpu, cpu, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    monkeypatch.setattr(lib, "_current", lambda stream: (None, -1))                  # as if the CPU were the current device
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    with pytest.raises(ValueError, match="axis_of_pair"):
        lib.rope(torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(32), axis_of_pair=[1] * 32)
    with pytest.raises(ValueError, match="int32"):
        lib.rope(torch.zeros(1, 1, 4, dtype=torch.int64), torch.zeros(32))
    r = lib.rope(torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(ValueError, match="positions"):
        lib.burst_attn_rope(lib.shape(1, 2, 2, 64, 5, 0, 1.0), r, cpu, cpu)
    with pytest.raises(ValueError, match="tensor of"):
        lib.burst_attn_rope(lib.shape(1, 3, 1, 64, 4, 0, 1.0), r, cpu, cpu)
    pages = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="scales"):
        lib.paged_cache(pages, pages, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), k_scale=torch.ones(3))
    cache = lib.paged_cache(pages, pages, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="another batch"):
        lib.burst_attn_decode(lib.shape(2, 2, 2, 64, 1, 16, 1.0), cache, cpu, cpu)
    with pytest.raises(ValueError, match="tensor of"):
        lib.burst_attn_rope(lib.shape(1, 2, 2, 64, 4, 0, 1.0), r, cpu, cpu[:0])
    with pytest.raises(ValueError, match="contiguous"):
        lib.burst_attn_rope(lib.shape(1, 2, 2, 64, 4, 0, 1.0), r, cpu, torch.zeros(1, 4, 64, 2).transpose(2, 3))
    with pytest.raises(ValueError, match="lse"):
        q = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16)
        lib.burst_attn_decode(lib.shape(1, 2, 2, 64, 1, 16, 1.0), cache, q, q, lse=torch.zeros(1, 2, 2))


def test_quotients_by_the_page_size(lib):
    """The kernels' division by a page's rows, restated: n * ceil(2^(31+s) / d) / 2^(31+s) is n / d for all n below 2^31."""
    for d in list(range(2, 300)) + [1 << k for k in range(1, 21)] + [(1 << 20) - 1, 65537, 48, 1000003]:
        s = (d - 1).bit_length()
        m = -(-(1 << (31 + s)) // d)
        assert m < 1 << 32
        for n in {0, 1, d - 1, d, d + 1, (1 << 30) // d * d - 1, (1 << 30) // d * d, (1 << 31) - 1, ((1 << 31) - 1) // d * d, ((1 << 31) - 1) // d * d - 1}:
            if n >= 0:
                assert (n * m >> 32) >> (s - 1) == n // d
