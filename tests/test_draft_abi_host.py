"""Attention of drafted tokens, pages and rows that move, and scores at the C-ABI boundary and in the binding, on the CPU: struct layouts, and that what the interface
rules out is refused before anything could reach a GPU (the addresses are made up and never dereferenced)."""
import ctypes as C

import pytest

from tests import test_cache_abi_host as base
from tests.test_cache_binding_host import OnDevice, calls as recorded  # noqa: F401  (a fixture)

INF, NAN = float("inf"), float("nan")


class Calls(base.Calls):
    def __init__(self, lib):
        super().__init__(lib)
        self.plan = lib.burst_tree_t(0x8000, 5, 0x9000, 5, 0xa000, 4, 0)

    def tree(self, ws=0x700000, ws_bytes=1 << 40, **kw):
        a = dict(shape=self.shape(), cache=self.cache, tree=self.plan, q=self.t, o=self.tensor(0x20000), lse=self.lib.burst_rowvec_t(0x30000, 40, 5))
        a.update(kw)
        return self.raw.burst_attn_tree(*[self.ref(a[n]) for n in ("shape", "cache", "tree", "q", "o", "lse")], ws, ws_bytes, None)

    def layers(self, n=3, first=None, **kw):
        """Caches of n layers, each at places of its own; kw replaces fields of the last."""
        first = first or self.cache
        at = lambda t, i: self.changed(t, ptr=t.ptr + (i << 32))
        caches = [self.changed(first, k=at(first.k, i), v=at(first.v, i)) for i in range(n)]
        caches[-1] = self.changed(caches[-1], **kw)
        return (self.lib.burst_cache_t * n)(*caches)

    def copy(self, shape=None, n=None, caches=None, moves=0xb000, n_moves=7):
        caches = self.layers() if caches is None else caches
        return self.raw.burst_attn_cache_copy_pages(C.byref(shape or self.shape()), len(caches) if n is None else n, caches, moves, n_moves, None)

    def keep(self, shape=None, n=None, caches=None, source=0xb000, stride=5, new=0xc000, kept=0xd000):
        caches = self.layers() if caches is None else caches
        return self.raw.burst_attn_cache_keep_rows(C.byref(shape or self.shape()), len(caches) if n is None else n, caches, source, stride, new, kept, None)


class ScoreCalls:
    def __init__(self, lib):
        self.lib, self.raw = lib, lib.raw()

    def shape(self, n_tokens=5, vocab=1000, n_top=3, scale=1.0):
        return self.lib.burst_scores_shape_t(n_tokens, vocab, n_top, scale)

    def scores(self, shape="", **kw):
        a = dict(logits=0x1000, dtype=1, ld=1000, y=0x2000, logp=0x3000, lse=0x4000, entropy=0x5000, top_logp=0x6000, top_ids=0x7000, ws=0x10000, ws_bytes=1 << 40)
        a.update(kw)
        shape = self.shape() if shape == "" else shape
        return self.raw.burst_lm_head_scores(None if shape is None else C.byref(shape), *a.values(), None)

    def bwd(self, shape="", **kw):
        a = dict(logits=0x1000, dtype=1, ld=1000, y=0x2000, lse=0x4000, entropy=0x5000, top_ids=0x7000, g_logp=0x8000, g_lse=0x9000, g_entropy=0xa000, g_top=0xb000,
                 d_logits=0xc0000, d_dtype=0, ld_d=1008)
        a.update(kw)
        shape = self.shape() if shape == "" else shape
        return self.raw.burst_lm_head_scores_bwd(None if shape is None else C.byref(shape), *a.values(), None)


@pytest.fixture
def calls(lib):
    return Calls(lib)


@pytest.fixture
def score_calls(lib):
    return ScoreCalls(lib)


def test_struct_layouts_match_the_header(lib):
    assert C.sizeof(lib.burst_tree_t) == 48 and lib.burst_tree_t.sink_rows.offset == 40 and lib.burst_tree_t.tokens.offset == 32
    assert C.sizeof(lib.burst_scores_shape_t) == 24 and lib.burst_scores_shape_t.scale.offset == 20


def test_tree_refusals(lib, calls):
    INV, UNS, c = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, calls
    base._cache_refusals(lib, c, lambda shape=None, **kw: c.tree(shape=shape or c.shape(), **kw))
    assert c.tree(shape=c.shape(sq=0)) == INV and c.tree(shape=c.shape(sq=-1)) == INV and c.tree(shape=c.shape(sq=65)) == UNS
    assert c.tree(shape=c.shape(sk=2049)) == INV and c.tree(shape=c.shape(head_dim=32)) == UNS and c.tree(shape=c.shape(scale=INF)) == INV
    far = c.tensor(0x20000, strides=(1 << 14, 1 << 12, 128))
    assert c.tree(shape=c.shape(batch=1 << 21), o=far) == UNS                          # 2^21 sequences * 8 heads * 5 tokens
    assert c.tree(q=None) == INV and c.tree(o=None) == INV and c.tree(q=c.tensor(dtype=1)) == UNS and c.tree(tree=None) == INV
    assert c.tree(o=c.tensor(0x20000, strides=(0, 1 << 12, 128))) == INV
    assert c.tree(lse=lib.burst_rowvec_t(0x30002, 40, 5)) == INV and c.tree(lse=lib.burst_rowvec_t(0x30000, 40, 4)) == INV
    for name, value in (("sink_rows", -1), ("seen", 0x8004), ("first_row", 0x9002), ("tokens", 0xa001), ("seen_stride", 4), ("seen_stride", -5),
                        ("first_stride", 4), ("first_stride", 1 << 59)):
        assert c.tree(tree=c.changed(c.plan, **{name: value})) == INV, name
    raw = lib.raw()
    need = lib.burst_attn_tree_workspace_bytes(c.shape(sq=8, batch=1, sk=1 << 20))
    assert need > 0
    large = c.changed(c.cache, table_cols=1 << 14, table_stride=1 << 14)
    shape, tree = c.shape(sq=8, batch=1, sk=1 << 20), lib.burst_tree_t(None, 0, None, 0, None, 0, 0)
    lse = lib.burst_rowvec_t(0x30000, 64, 8)
    for bad in (dict(ws=None), dict(ws=0x700010), dict(ws_bytes=need - 1)):
        assert c.tree(shape=shape, cache=large, tree=tree, lse=lse, **bad) == INV
    for bad in (c.shape(sq=0), c.shape(sq=65), c.shape(q_heads=9), c.shape(sk=-1), c.shape(head_dim=256)):
        assert raw.burst_attn_tree_workspace_bytes(C.byref(bad)) == -1
        assert raw.burst_attn_tree_plan(C.byref(bad), (C.c_int32 * 3)()) in (INV, UNS)
    assert raw.burst_attn_tree_workspace_bytes(None) == -1 and raw.burst_attn_tree_plan(C.byref(c.shape()), None) == INV


@pytest.mark.parametrize("which", ["copy", "keep"])
def test_refusals_of_moves(lib, calls, which):
    INV, UNS, c = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, calls
    call = getattr(c, which)
    base._cache_refusals(lib, c, lambda shape=None, cache=0: call(shape=shape) if cache == 0 else call(caches=None, n=0) if cache is None else
                         call(caches=(lib.burst_cache_t * 1)(cache)))
    assert call(n=0) == INV and call(n=-1) == INV and call(n=1025, caches=c.layers(1025)) == UNS
    raw_call = c.raw.burst_attn_cache_copy_pages if which == "copy" else c.raw.burst_attn_cache_keep_rows
    rest = (0xb000, 7, None) if which == "copy" else (0xb000, 5, 0xc000, 0xd000, None)
    assert raw_call(C.byref(c.shape()), 1, None, *rest) == INV
    other = c.tensor(c.cache.k.ptr + (2 << 32), 0, (1 << 17, 1 << 10, 128)), c.tensor(c.cache.v.ptr + (2 << 32), 0, (1 << 17, 1 << 10, 128))
    for bad in (dict(n_pages=99), dict(page_rows=128), dict(k=other[0], v=other[1]), dict(k=c.cache.k), dict(v=c.layers()[2].k)):
        assert call(caches=c.layers(**bad)) == INV, bad
    over = (1 << 15, 1 << 10, 128)                                                     # a page's 64 rows reach into the next page
    assert call(caches=c.layers(first=c.changed(c.cache, k=c.tensor(0x100000, 0, over), v=c.tensor(0x900000, 0, over)))) == INV
    if which == "copy":
        assert call(moves=None) == INV and call(moves=0xb002) == INV and call(n_moves=-1) == INV and call(n_moves=1 << 31) == UNS
        assert call(moves=None, n_moves=0) == lib.BURST_OK                             # nothing to do
        return
    for bad in (dict(table=0x3100), dict(table_cols=31), dict(table_stride=33), dict(rows=0x4100)):
        assert call(caches=c.layers(**bad)) == INV, bad
    assert call(source=None) == INV and call(source=0xb001) == INV and call(kept=None) == INV and call(kept=0xd002) == INV and call(new=0xc002) == INV
    assert call(stride=4) == INV and call(stride=-1) == INV and call(shape=c.shape(sq=65)) == UNS and call(shape=c.shape(sq=-1)) == INV
    assert call(shape=c.shape(sq=0), source=None, kept=None, new=None) == lib.BURST_OK


@pytest.mark.parametrize("which", ["scores", "bwd"])
def test_scores_refusals(lib, score_calls, which):
    INV, UNS, c = lib.BURST_ERR_INVALID_ARG, lib.BURST_ERR_UNSUPPORTED, score_calls
    call = getattr(c, which)
    assert call(None) == INV
    for status, shape in ((INV, dict(n_tokens=-1)), (INV, dict(vocab=0)), (INV, dict(n_top=-1)), (INV, dict(vocab=2)), (INV, dict(scale=0.0)), (INV, dict(scale=-1.0)),
                          (INV, dict(scale=INF)), (INV, dict(scale=NAN)), (UNS, dict(n_top=65)), (UNS, dict(vocab=(1 << 30) + 1)), (UNS, dict(n_tokens=(1 << 25) + 1))):
        shape = c.shape(**shape)
        assert call(shape) == status
        assert c.raw.burst_lm_head_scores_workspace_bytes(C.byref(shape)) == -1 and c.raw.burst_lm_head_scores_plan(C.byref(shape), (C.c_int32 * 2)()) == status
    for bad in (dict(dtype=2), dict(dtype=-1), dict(ld=999), dict(ld=(1 << 34) + 1), dict(logits=None), dict(logits=0x1008), dict(y=0x2004), dict(top_ids=0x7004)):
        assert call(**bad) == INV, bad
    assert c.raw.burst_lm_head_scores_workspace_bytes(None) == -1 and c.raw.burst_lm_head_scores_plan(C.byref(c.shape()), None) == INV
    none = c.shape(n_tokens=0)
    if which == "scores":
        for bad in (dict(y=None), dict(logp=None), dict(logp=0x3002), dict(lse=0x4001), dict(entropy=0x5002), dict(top_logp=0x6003)):
            assert call(**bad) == INV, bad
        assert call(y=None, logp=None, lse=None, entropy=None, top_logp=None, top_ids=None) == INV
        assert call(c.shape(n_top=0)) == INV                                           # words wanted, none asked for
        long = c.shape(n_tokens=2, vocab=1 << 20)
        need = c.raw.burst_lm_head_scores_workspace_bytes(C.byref(long))
        assert need > 0
        for bad in (dict(ws=None), dict(ws=0x10080), dict(ws_bytes=need - 1)):
            assert call(long, ld=1 << 20, **bad) == INV, bad
        assert call(none, logits=None, y=None, logp=None, lse=None, entropy=None, top_logp=None, top_ids=None, ws=None, ws_bytes=0) == lib.BURST_OK
        return
    for bad in (dict(lse=None), dict(y=None), dict(entropy=None), dict(top_ids=None), dict(g_logp=0x8002), dict(g_lse=0x9001), dict(g_entropy=0xa002), dict(g_top=0xb003),
                dict(d_logits=None), dict(d_logits=0xc0004), dict(d_dtype=2), dict(ld_d=999), dict(d_logits=0x1000), dict(d_logits=0x1000, d_dtype=1)):
        assert call(**bad) == INV, bad
    assert call(g_logp=None, g_lse=None, g_entropy=None, g_top=None) == INV
    assert call(c.shape(n_top=0)) == INV
    assert call(none, logits=None, d_logits=None, lse=None) == lib.BURST_OK


def test_grids_and_sizes_of_the_largest(lib):
    """A launch of the scores has fewer than 2^32 threads: four rows for a work-group of 256, or a work-group of 64 threads a wave for each part of a row."""
    for n in (1, 2, 255, 256, 257, 2047, 2048, (1 << 23) - 1, 1 << 23, 1 << 25):
        for v in (1, 2048, 2049, 16383, 16384, 65535, 65536, 98304, 1 << 20, 1 << 30):
            waves, parts = lib.burst_lm_head_scores_plan(lib.scores_shape(n, v))
            threads = -(-n // 4) * 256 if waves == 1 else n * parts * 64 * waves
            assert threads < 1 << 32 and 1 <= parts <= 16 and (parts == 1 or waves == 16)
            assert (lib.burst_lm_head_scores_workspace_bytes(lib.scores_shape(n, v, min(v, 64))) > 0) == (parts > 1)


def _cache(lib, batch=2):
    import torch
    pages = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    return lib.paged_cache(pages, torch.zeros_like(pages), torch.zeros(batch, 1, dtype=torch.int32), torch.ones(batch, dtype=torch.int32))


def test_the_binding_refuses(lib, recorded):   # noqa: F811
    import torch
    i32, i64 = torch.int32, torch.int64
    cache = _cache(lib)
    q, shp = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), lib.shape(2, 4, 2, 64, 3, 16, 1.0)
    plan = lib.tree(torch.zeros(2, 3, dtype=i64), torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32), 2)
    assert (plan.seen_stride, plan.first_stride, plan.sink_rows, plan.elsewhere) == (3, 3, 2, 0)
    one = lib.tree(torch.zeros(1, 3, dtype=i64).expand(2, 3))
    assert one.seen_stride == 0
    lib.burst_attn_tree(shp, cache, plan, q, q)
    lib.burst_attn_tree(shp, cache, lib.tree(), q, q)
    bad_trees = (dict(seen=torch.zeros(2, 3, dtype=i32)), dict(seen=torch.zeros(3, dtype=i64)), dict(first_row=torch.zeros(2, 3, dtype=i64)),
                 dict(tokens=torch.zeros(2, 1, dtype=i32)), dict(seen=torch.zeros(3, 2, dtype=i64).T), dict(tokens=torch.zeros(4, dtype=i32)[::2]))
    for bad in bad_trees:
        with pytest.raises(ValueError, match="expected"):
            lib.tree(**bad)
    with pytest.raises(ValueError, match="expected"):
        lib.tree(torch.zeros(2, 3, dtype=i64), torch.zeros(2, 4, dtype=i32))
    with pytest.raises(ValueError, match="the tree is of"):
        lib.burst_attn_tree(shp, cache, lib.tree(torch.zeros(2, 4, dtype=i64)), q, q)
    with pytest.raises(ValueError, match="the tree is of"):
        lib.burst_attn_tree(shp, cache, lib.tree(tokens=torch.zeros(3, dtype=i32)), q, q)
    with pytest.raises(ValueError, match="lse"):
        lib.burst_attn_tree(shp, cache, plan, q, q, lse=torch.zeros(2, 3, 4))
    with pytest.raises(ValueError, match="another batch"):
        lib.burst_attn_tree(shp, _cache(lib, 1), plan, q, q)
    with pytest.raises(ValueError, match="tensor of"):
        lib.burst_attn_tree(shp, cache, plan, q[:, :2], q)
    layers = lib.cache_layers([cache, _cache(lib)])
    assert len(layers) == 2
    lib.burst_attn_cache_copy_pages(layers, torch.zeros(5, 3, dtype=i32))
    lib.burst_attn_cache_keep_rows(layers, torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32))
    for bad in ([], [cache, _cache(lib, 1)]):
        with pytest.raises(ValueError, match="caches"):
            lib.cache_layers(bad)
    for bad in (torch.zeros(5, 3, dtype=i64), torch.zeros(5, 2, dtype=i32), torch.zeros(15, dtype=i32), torch.zeros(3, 5, dtype=i32).T):
        with pytest.raises(ValueError, match="moves"):
            lib.burst_attn_cache_copy_pages(layers, bad)
    for source, kept in ((torch.zeros(3, 3, dtype=i32), torch.zeros(2, dtype=i32)), (torch.zeros(2, 3, dtype=i64), torch.zeros(2, dtype=i32)),
                         (torch.zeros(2, 3, dtype=i32), torch.zeros(3, dtype=i32))):
        with pytest.raises(ValueError):
            lib.burst_attn_cache_keep_rows(layers, source, kept)
    s, x = lib.scores_shape(4, 10, 2), torch.zeros(4, 10)
    f = torch.zeros(4)
    lib.burst_lm_head_scores(s, x, lse=f)
    lib.burst_lm_head_scores_bwd(s, x, f, x, g_lse=f)
    for bad in (dict(logits=torch.zeros(4, 11)), dict(logits=torch.zeros(10, 4).T), dict(lse=torch.zeros(4, dtype=torch.float64)), dict(lse=torch.zeros(4, 1)),
                dict(top_ids=torch.zeros(4, 2, dtype=i32)), dict(top_logp=torch.zeros(4, 3)), dict(y=torch.zeros(4, dtype=i32), logp=f)):
        with pytest.raises(ValueError, match="expected"):
            lib.burst_lm_head_scores(s, **{"logits": x, "lse": f, **bad})
    for bad in (dict(d_logits=torch.zeros(4, 9)), dict(g_top=torch.zeros(2, 4)), dict(g_lse=torch.zeros(8)[::2])):
        with pytest.raises(ValueError, match="expected"):
            lib.burst_lm_head_scores_bwd(s, **{"logits": x, "lse": f, "d_logits": x, "g_lse": f, **bad})
    assert [name for name, _ in recorded.made] == ["burst_attn_tree"] * 2 + ["burst_attn_cache_copy_pages", "burst_attn_cache_keep_rows", "burst_lm_head_scores",
                                                                           "burst_lm_head_scores_bwd"]


def test_what_lies_on_another_device_is_refused(lib, recorded, monkeypatch):   # noqa: F811
    import torch
    cache, plan = _cache(lib), lib.tree()
    layers = lib.cache_layers([cache])
    q, shp = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16), lib.shape(2, 4, 2, 64, 3, 16, 1.0)
    moves, source, kept = torch.zeros(5, 3, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    s, x, f = lib.scores_shape(4, 10), torch.zeros(4, 10), torch.zeros(4)
    far = OnDevice
    for call in (lambda: lib.burst_attn_tree(shp, cache, plan, far(q), q), lambda: lib.burst_attn_tree(shp, cache, plan, q, q, workspace=far(f)),
                 lambda: lib.tree(tokens=far(kept)), lambda: lib.burst_attn_cache_copy_pages(layers, far(moves)),
                 lambda: lib.burst_attn_cache_keep_rows(layers, far(source), kept), lambda: lib.burst_lm_head_scores(s, far(x), lse=f)):
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.setattr(lib, "_current", lambda stream: (None, 1))
    for call in (lambda: lib.burst_attn_tree(shp, cache, plan, far(q), far(q)), lambda: lib.burst_attn_cache_copy_pages(layers, far(moves)),
                 lambda: lib.burst_attn_cache_keep_rows(layers, far(source), far(kept)), lambda: lib.burst_lm_head_scores_bwd(s, far(x), f, far(x), g_lse=f)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert recorded.made == []
