"""Appending to a paged cache, attention of one new token over it, and the two together, on the GPU against the fp64 reference.

Tolerances of the attention, with u = 2^-24 and A the largest sum of |q| |K| of a head times the scale: a score is a sum of head_dim
exact products in fp32, off by at most head_dim u A, and its conversion to base 2 by 4 u A.  So Lse is off by at most e = (head_dim + 4) u A, and
(n + 16) u for the sum of n numbers, exponential and logarithm, and 4 u of its own size; O by (2 e + (n + 16) u + 2^-16) sum P |V|, where 2^-16 covers P as a
sum of two bf16 numbers (a truncated one and a rounded rest: 2^-8 * 2^-9 of it, doubled), and half a step of its type."""
import math

import numpy as np
import pytest

from oracle import burst_oracle as oc
from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import helpers as hp
from tests import test_gpu_rope as tr

pytestmark = pytest.mark.gpu


class Paged:
    """A cache with random contents and a random table, on both sides.  by_head: heads outside rows in memory."""

    def __init__(self, lib, rng, rows, page_rows, Hkv, d, f8=False, by_head=False, spare=2, cols=None, fill=None):
        import torch
        self.rows, self.page_rows, self.f8 = list(rows), page_rows, f8
        pages = [-(-max(r, 0) // page_rows) for r in rows]
        self.n_pages = sum(pages) + spare
        cols = cols or max(max(pages), 1)
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(rows), cols), -7, np.int32)
        at = 0
        for b, p in enumerate(pages):
            self.table[b, :p] = order[at:at + p]
            at += p
        shape = (self.n_pages, page_rows, Hkv, d)
        dtype = torch.float8_e4m3fn if f8 else torch.bfloat16
        self.k_scale = rng.uniform(0.005, 0.02, Hkv).astype(np.float32) if f8 else None
        self.v_scale = rng.uniform(0.005, 0.02, Hkv).astype(np.float32) if f8 else None
        self.dev, self.host = {}, {}
        for name in "kv":
            x = rng.standard_normal(shape, dtype=np.float32) * (96.0 if f8 else 1.0) if fill is None else np.full(shape, fill, np.float32)
            mem = torch.empty((self.n_pages, Hkv, page_rows, d) if by_head else shape, device="cuda", dtype=dtype)
            t = mem.transpose(1, 2) if by_head else mem
            t.copy_(torch.from_numpy(np.clip(x, -448, 448) if f8 else x).to(dtype))
            self.dev[name], self.host[name] = t, t.float().cpu().numpy().astype(np.float64)
        put = lambda a: None if a is None else torch.from_numpy(a).cuda()
        self.put_table, self.put_rows = put(self.table), put(np.array(rows, np.int32))
        self.cache = lib.paged_cache(self.dev["k"], self.dev["v"], self.put_table, self.put_rows, put(self.k_scale), put(self.v_scale))

    def refresh(self):
        """The host's copy of what the GPU holds."""
        for name in "kv":
            self.host[name] = self.dev[name].float().cpu().numpy().astype(np.float64)

    def decode(self, q, scale, first=None, max_rows=None, rows=None):
        return co.decode(q, self.host["k"], self.host["v"], self.table, rows or self.rows, scale, first, max_rows, self.k_scale, self.v_scale)


def run_decode(lib, P, q, scale, max_rows, first=None, o_type="f32", want_lse=True, ws=None):
    import torch
    B, Hq, d = q.shape[0], q.shape[2], q.shape[3]
    shp = lib.shape(B, Hq, P.dev["k"].size(2), d, 1, max_rows, scale)
    o = torch.full((B, 1, Hq, d), 7.0, device="cuda", dtype=torch.float32 if o_type == "f32" else torch.bfloat16)
    lse = torch.full((B, Hq, 1), 7.0, device="cuda") if want_lse else None
    if ws is None:
        ws = torch.full((lib.burst_attn_decode_workspace_bytes(shp),), 255, device="cuda", dtype=torch.uint8)   # NaN everywhere
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    lib.burst_attn_decode(shp, P.cache, q, o, lse, ws, first_row=f)
    torch.cuda.synchronize()
    return o, lse


def check_decode(o, lse, ref, n, d, bf16=False):
    O, lse_ref, weight, size = ref
    u = 2.0 ** -24
    e = (d + 4) * u * size
    got = o.double().cpu().numpy()[:, 0]
    tol = (2 * e + (n + 16) * u + 2.0 ** -16)[..., None] * weight
    if bf16:
        tol = tol + 2.0 ** -8 * np.maximum(np.abs(O) + tol, 2.0 ** -126)
    assert (np.abs(got - O) <= tol).all(), float((np.abs(got - O) - tol).max())
    dead = lse_ref == -np.inf
    assert (got[dead] == 0).all()
    if lse is not None:
        l = lse.double().cpu().numpy()[..., 0]
        assert (l[dead] == -np.inf).all()
        assert (np.abs(l[~dead] - lse_ref[~dead]) <= (e + (n + 16) * u + 4 * u * np.abs(lse_ref))[~dead]).all()


def queries(rng, B, Hq, d):
    bits = wl.f32_to_bf16_bits(rng.standard_normal((B, 1, Hq, d), dtype=np.float32))
    return hp.dev_bf16(bits), hp.widen(bits)[:, 0]


DECODES = [
    # rows, first rows, page rows, q_heads, kv_heads, head_dim, e4m3, by head, type of O
    ([1], None, 16, 1, 1, 64, False, False, "f32"),
    ([777], None, 16, 12, 12, 64, False, False, "bf16"),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65], None, 16, 8, 2, 128, False, False, "f32"),
    ([127, 128, 129, 255, 256, 257, 0, 500], None, 32, 8, 8, 128, False, True, "f32"),
    ([1000, 3, 2049], [990, 3, 1], 64, 16, 1, 128, False, False, "f32"),
    ([300, 300, 300, 300], [-5, 299, 300, 2 ** 31 - 1], 48, 6, 2, 64, False, True, "bf16"),
    ([400, 17], None, 1, 4, 4, 128, False, False, "f32"),
    ([400, 17, 161], [7, 0, 160], 5, 9, 3, 64, False, False, "f32"),
    ([5000], None, 256, 17, 1, 128, False, False, "f32"),
    ([333, 1111], None, 16, 66, 2, 128, False, False, "f32"),
    ([200, 1500], [13, 77], 24, 32, 1, 64, False, False, "f32"),
    ([700], None, 16, 64, 1, 64, False, True, "bf16"),
    ([1, 130, 0, 999], None, 16, 8, 8, 128, True, False, "f32"),
    ([2500, 40], [100, 39], 64, 64, 8, 128, True, True, "bf16"),
    ([333, 96], None, 16, 5, 5, 64, True, False, "f32"),
    ([77, 1025], [5, 1000], 7, 40, 1, 128, True, False, "f32"),
    ([129, 64, 1], None, 3, 6, 3, 64, True, True, "f32"),
]


@pytest.mark.parametrize("case", DECODES)
def test_decode_against_the_reference(lib, case):
    rows, first, page_rows, Hq, Hkv, d, f8, by_head, o_type = case
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 82000 + sum(rows) + Hq))
    P = Paged(lib, rng, rows, page_rows, Hkv, d, f8, by_head)
    q, q_host = queries(rng, len(rows), Hq, d)
    print(f"decode {case}", flush=True)
    # the bound: the longest sequence's rows, and what the table could name
    for max_rows in sorted({max(rows), P.table.shape[1] * page_rows}):
        o, lse = run_decode(lib, P, q, d ** -0.5, max_rows, first, o_type)
        check_decode(o, lse, P.decode(q_host, d ** -0.5, first), max(rows), d, o_type == "bf16")
    o2, _ = run_decode(lib, P, q, d ** -0.5, max(rows), first, o_type, want_lse=False)
    o, _ = run_decode(lib, P, q, d ** -0.5, max(rows), first, o_type)
    assert o.equal(o2)                                                     # the same call, the same bits, with Lse and without


@pytest.mark.parametrize("d,f8", [(128, False), (64, True)])
def test_long_sequence_of_one_head(lib, d, f8):
    """Split over as many work-groups as there are: 40000 rows of one sequence."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 82500))
    P = Paged(lib, rng, [40001], 64, 1, d, f8)
    q, q_host = queries(rng, 1, 3, d)
    o, lse = run_decode(lib, P, q, d ** -0.5, 40001)
    check_decode(o, lse, P.decode(q_host, d ** -0.5), 40001, d)


def test_many_sequences(lib):
    """More sequences than a work-group has threads, of 0 to 200 rows, with one long one among them."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 82600))
    rows = rng.integers(0, 200, 700).tolist()
    rows[333], rows[0], rows[699] = 3000, 0, 1
    P = Paged(lib, rng, rows, 16, 2, 64)
    q, q_host = queries(rng, 700, 4, 64)
    o, lse = run_decode(lib, P, q, 0.125, 3000)
    check_decode(o, lse, P.decode(q_host, 0.125), 3000, 64)


def test_all_empty(lib):
    rng = np.random.Generator(np.random.PCG64(3))
    P = Paged(lib, rng, [0, 0, -4], 16, 2, 128, cols=4)
    q, q_host = queries(rng, 3, 4, 128)
    for max_rows in (0, 1, 64):
        o, lse = run_decode(lib, P, q, 0.1, max_rows)
        assert (o == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("page_rows", [16, 5])
def test_pages_that_are_none_and_rows_beyond_the_bound(lib, page_rows):
    """Entries of the table outside the cache hide their rows; so does the bound; nothing else changes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 82700 + page_rows))
    rows = [200, 200, 170, 10 ** 6]
    P = Paged(lib, rng, [200, 200, 170, 200], page_rows, 2, 128)
    P.table[0, 3], P.table[1, :] = P.n_pages, -1
    P.table[2, 0], P.table[2, -1] = 2 ** 31 - 1, -2 ** 31
    P.put_table.copy_(torch.from_numpy(P.table))
    P.put_rows.copy_(torch.tensor(rows, dtype=torch.int32))               # the last one: as many as the table has room for
    q, q_host = queries(rng, 4, 4, 128)
    for max_rows in (200, 130, 33, 1):
        o, lse = run_decode(lib, P, q, 0.09, max_rows)
        ref = P.decode(q_host, 0.09, max_rows=max_rows, rows=rows)
        assert (ref[1][1] == -np.inf).all()
        check_decode(o, lse, ref, 200, 128)


@pytest.mark.parametrize("f8,page_rows", [(False, 16), (False, 6), (True, 32)])
def test_what_is_not_seen_may_hold_anything(lib, f8, page_rows):
    """NaN and infinities in every row of the cache that no sequence sees: behind the last row, before the first, in spare pages."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 82800 + page_rows))
    rows, first = [100, 37, 16, 161], [33, 0, 15, 150]
    P = Paged(lib, rng, rows, page_rows, 2, 64, f8)
    seen = np.zeros((P.n_pages, page_rows), bool)
    for b in range(4):
        page, r = co.slots(P.table, page_rows, b, np.arange(first[b], rows[b]))
        seen[page, r] = True
    hidden = torch.from_numpy(~seen).cuda()
    for name, bad in (("k", float("nan")), ("v", float("nan") if f8 else float("inf"))):
        P.dev[name].view(torch.uint8 if f8 else torch.bfloat16)[hidden] = 0x7f if f8 else bad
    q, q_host = queries(rng, 4, 6, 64)
    o, lse = run_decode(lib, P, q, 0.125, 161, first)
    check_decode(o, lse, P.decode(q_host, 0.125, first), 161, 64)


def test_infinities_and_nan_that_are_seen(lib):
    """A NaN key makes its heads' results NaN, a value's infinity its element's; a key at -inf towards the query has no share."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 82900))
    P = Paged(lib, rng, [300], 16, 3, 64)
    q, q_host = queries(rng, 1, 6, 64)
    page, r = co.slots(P.table, 16, 0, 123)
    P.dev["k"][page, r, 0, 5] = float("nan")
    P.dev["v"][page, r, 1, 7] = float("inf")
    P.dev["k"][page, r, 2, 9] = -math.inf if q_host[0, 4, 9] > 0 else math.inf       # -inf for head 4
    o, lse = run_decode(lib, P, q, 0.125, 300)
    assert torch.isnan(o[0, 0, :2]).all() and torch.isnan(lse[0, :2]).all()
    assert (o[0, 0, 2:4, 7] == math.inf).all() and torch.isfinite(o[0, 0, 2:4, :7]).all() and torch.isfinite(lse[0, 2:4]).all()
    P.host["k"][page, r, 2], P.host["v"][page, r, 1], P.host["k"][page, r, 0] = 0, 0, 0
    keep = [t for t in range(300) if t != 123]
    gather = lambda x: x[co.slots(P.table, 16, 0, np.array(keep))]
    s = gather(P.host["k"])[:, 2] @ q_host[0, 4] * 0.125
    p = np.exp(s - s.max())
    assert np.abs(o[0, 0, 4].double().cpu().numpy() - p @ gather(P.host["v"])[:, 2] / p.sum()).max() <= 1e-4
    assert abs(lse[0, 4].item() - (s.max() + np.log(p.sum()))) <= 1e-4


def test_scores_of_all_sizes(lib):
    """Scores that grow from row to row, that fall, and far below zero: the running maximum follows; nothing overflows or vanishes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 83000))
    rows = [1000, 1000, 1000, 1000]
    P = Paged(lib, rng, rows, 16, 1, 64, fill=0.0)
    ramp = np.linspace(-600.0, 600.0, 1000)
    for b, s in enumerate((ramp, ramp[::-1], np.full(1000, -700.0), np.where(np.arange(1000) == 517, 900.0, -900.0))):
        page, r = co.slots(P.table, 16, b, np.arange(1000))
        P.dev["k"][page, r, 0, 0] = torch.from_numpy(s.copy()).to(torch.bfloat16).cuda()
        P.dev["v"][page, r, 0] = torch.randn(1000, 64, device="cuda").to(torch.bfloat16)
    P.refresh()
    q = torch.zeros(4, 1, 2, 64, device="cuda", dtype=torch.bfloat16)
    q[:, :, 0, 0], q[:, :, 1, 0] = 1.0, -1.0
    o, lse = run_decode(lib, P, q, 1.0, 1000)
    check_decode(o, lse, P.decode(q.double().cpu().numpy()[:, 0], 1.0), 1000, 64)


def test_offsets_beyond_32_bits(lib):
    """Pages up to 3 GiB and heads 4 GiB from each other."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 83100))
    page, head, n_pages, d = 64 * 128, 1 << 31, 4, 128                    # (elements)
    flat = torch.empty(2 * head, device="cuda", dtype=torch.bfloat16)
    x = flat.as_strided((n_pages, 64, 2, d), (1 << 29, d, head, 1))[1:4]   # (pages 1 GiB apart)
    k = torch.empty(3, 64, 2, d).normal_(generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    x.copy_(k)
    v = flat[page:].as_strided((n_pages, 64, 2, d), (1 << 29, d, head, 1))[1:4]
    w = torch.empty(3, 64, 2, d).normal_(generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    v.copy_(w)
    table, rows = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([150], dtype=torch.int32, device="cuda")
    q, q_host = queries(rng, 1, 4, d)
    o, lse = torch.empty(1, 1, 4, d, device="cuda"), torch.empty(1, 4, 1, device="cuda")
    shp = lib.shape(1, 4, 2, d, 1, 192, 0.09)
    ws = torch.empty(lib.burst_attn_decode_workspace_bytes(shp), device="cuda", dtype=torch.uint8)
    lib.burst_attn_decode(shp, lib.paged_cache(x, v, table, rows), q, o, lse, ws)
    wide = lambda t: t.float().numpy().astype(np.float64)
    check_decode(o, lse, co.decode(q_host, wide(k), wide(w), table.cpu().numpy(), [150], 0.09), 150, d)
    # and an append there
    new = torch.randn(1, 3, 2, d, device="cuda").to(torch.bfloat16)
    lib.burst_attn_cache_append(lib.shape(1, 4, 2, d, 3, 0, 1.0), lib.paged_cache(x, v, table, rows), new, new)
    assert torch.equal(x[1, 19:22], new[0]) and torch.equal(v[1, 19:22], new[0])


def test_a_row_does_not_depend_on_its_batch(lib):
    """The same sequence alone and among others: other roundings in fp32 (S minus another maximum, sums in another order), 2^-20 of O at most."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 83200))
    rows = [1777, 5, 900, 3100, 64, 1777]
    P = Paged(lib, rng, rows, 16, 2, 128)
    q, _ = queries(rng, 6, 8, 128)
    o, lse = run_decode(lib, P, q, 0.09, 3100)
    alone = lib.paged_cache(P.dev["k"], P.dev["v"], P.put_table[:1], P.put_rows[:1])
    P.cache = alone
    o1, lse1 = run_decode(lib, P, q[:1], 0.09, 1777)
    assert (o1[0] - o[0]).abs().max() <= 2.0 ** -20 * o[0].abs().max() + 2.0 ** -24
    assert (lse1[0] - lse[0]).abs().max() <= 2.0 ** -20


APPENDS = [
    # batch, new rows of each (None: all), rows, page rows, q_heads, kv_heads, head_dim, rotary_dim, e4m3, by head
    (1, None, [1], 16, 1, 1, 64, 64, False, False, 1),
    (3, [1, 1, 1], [1, 600, 77], 16, 32, 8, 128, 128, False, False, 1),
    (4, [0, 7, 33, 20], [5, 7, 100, 10], 16, 6, 2, 64, 32, False, True, 33),
    (2, [50, 64], [130, 64], 48, 5, 5, 128, 112, False, False, 64),
    (2, [70, 9], [70, 300], 7, 4, 1, 128, 128, True, False, 70),
    (3, [-3, 1000, 2], [20, 40, 4000], 16, 8, 4, 64, 64, True, True, 30),
    (2, None, [40, 41], 1, 2, 2, 128, 16, False, False, 40),
]


@pytest.mark.parametrize("case", APPENDS)
@pytest.mark.parametrize("adjacent", [False, True])
def test_append_against_the_reference(lib, case, adjacent):
    import torch
    B, new, rows, page_rows, Hq, Hkv, d, R, f8, by_head, n = case
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 84000 + sum(rows) + Hq))
    P = Paged(lib, rng, rows, page_rows, Hkv, d, f8, by_head)
    counts = [n] * B if new is None else [min(max(x, 0), n) for x in new]
    pos = rng.integers(0, 1 << 20, (2, B, n)).astype(np.int32)
    axes = rng.integers(0, 2, R // 2).tolist()
    freq = tr._frequencies(R // 2)
    rope = lib.rope(torch.from_numpy(pos).cuda(), torch.from_numpy(freq).cuda(), adjacent=adjacent, axis_of_pair=axes)
    bits = {name: wl.f32_to_bf16_bits(rng.standard_normal((B, n, h, d), dtype=np.float32)) for name, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    if f8:
        bits["v"][..., 3] = 0x4f80                                         # 2^32: beyond what e4m3 holds over these scales
    dev, host = {x: hp.dev_bf16(b) for x, b in bits.items()}, {x: hp.widen(b) for x, b in bits.items()}
    q_out = torch.full((B, n, Hq, d), 7.0, device="cuda", dtype=torch.bfloat16)
    before = dict(P.host)
    new_rows = None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda")
    print(f"append {case}", flush=True)
    lib.burst_attn_cache_append(lib.shape(B, Hq, Hkv, d, n, 0, 1.0), P.cache, dev["k"], dev["v"], new_rows, rope, dev["q"], q_out)
    torch.cuda.synchronize()
    P.refresh()
    turned = {x: co.rope(host[x], pos, freq, axes, adjacent) for x in "qk"}
    angle = co.angles(pos, freq, axes)
    got = q_out.double().cpu().numpy()
    tol = {x: tr.tolerance(host[x], turned[x], angle, R, adjacent, True) for x in "qk"}
    places = list(co.new_places(P.table, page_rows, P.n_pages, rows, counts))
    assert len(places) == sum(min(c, max(min(r, P.table.shape[1] * page_rows), 0)) for c, r in zip(counts, rows))
    for b in range(B):
        assert (np.abs(got[b, :counts[b]] - turned["q"][b, :counts[b]]) <= tol["q"][b, :counts[b]]).all()
        assert (got[b, counts[b]:] == 7.0).all()
    for name, x, scale in (("k", turned["k"], P.k_scale), ("v", host["v"], P.v_scale)):
        want, close = before[name].copy(), np.zeros_like(before[name])
        for b, i, page, r in places:
            if f8:
                want[page, r] = np.clip(x[b, i] / scale[:, None].astype(np.float64), -448, 448)
                # the rotated value's own error and two roundings of the division, then half a step of e4m3 (2^-10 at its bottom)
                own = (tr.tolerance(host["k"], turned["k"], angle, R, adjacent, False)[b, i] / scale[:, None] if name == "k" else 0.0)
                close[page, r] = own + 3 * 2.0 ** -24 * np.abs(want[page, r]) + np.maximum(2.0 ** -4 * (np.abs(want[page, r]) + own), 2.0 ** -10)
            else:
                want[page, r], close[page, r] = x[b, i], tol["k"][b, i] if name == "k" else 0.0
        assert (np.abs(P.host[name] - want) <= close).all()                # everything else in the cache: as it was


def test_append_without_rotation_keeps_bits(lib):
    import torch
    rng = np.random.Generator(np.random.PCG64(1))
    P = Paged(lib, rng, [20, 3], 16, 2, 64)
    k = torch.randint(-2 ** 15, 2 ** 15, (2, 3, 2, 64), device="cuda", dtype=torch.int16).view(torch.bfloat16)   # any bits
    k = torch.where(torch.isnan(k), torch.zeros_like(k), k)
    lib.burst_attn_cache_append(lib.shape(2, 2, 2, 64, 3, 0, 1.0), P.cache, k, k)
    for name in "kv":
        page, r = (torch.from_numpy(a).cuda() for a in co.slots(P.table, 16, 0, np.arange(17, 20)))
        assert torch.equal(P.dev[name][page, r].view(torch.int16), k[0].view(torch.int16))


def test_append_to_pages_that_are_none(lib):
    """Such rows are left out, their queries turned all the same; rows beyond the table too."""
    import torch
    rng = np.random.Generator(np.random.PCG64(2))
    P = Paged(lib, rng, [64, 64], 16, 1, 64)
    P.table[0, 2], P.table[1, 3] = -1, P.n_pages
    P.put_table.copy_(torch.from_numpy(P.table))
    P.put_rows.copy_(torch.tensor([64, 1000], dtype=torch.int32))          # taken as 64
    x = torch.randn(2, 40, 1, 64, device="cuda").to(torch.bfloat16)
    lib.burst_attn_cache_append(lib.shape(2, 1, 1, 64, 40, 0, 1.0), P.cache, x, x)
    before, host = dict(P.host), x.double().cpu().numpy()
    P.refresh()
    for name in "kv":
        assert np.array_equal(P.host[name], co.append(before[name], host, P.table, [64, 64], [40, 40]))


def test_nan_and_infinity_in_eight_bits(lib):
    import torch
    rng = np.random.Generator(np.random.PCG64(2))
    P = Paged(lib, rng, [1], 16, 1, 64, f8=True)
    x = torch.zeros(1, 1, 1, 64, device="cuda", dtype=torch.bfloat16)
    x[..., 0], x[..., 1], x[..., 2] = float("nan"), float("inf"), float("-inf")
    lib.burst_attn_cache_append(lib.shape(1, 1, 1, 64, 1, 0, 1.0), P.cache, x, x)
    page, r = co.slots(P.table, 16, 0, 0)
    for name in "kv":
        got = P.dev[name][page, r, 0].float()
        assert torch.isnan(got[0]) and got[1] == 448 and got[2] == -448 and (got[3:] == 0).all()


def test_tokens_one_after_the_other(lib):
    """As a model uses them: a prompt through the ring's forward pass and into the cache, then tokens one by one, each turned, appended and
    attended, from one captured graph that is replayed with the program's own updates between; against the attention oracle of the ring over the
    whole sequence."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 85000))
    B, Hq, Hkv, d, page_rows, steps = 2, 8, 2, 64, 16, 9
    lens = [45, 30]                                                        # the prompts
    scale, cols = d ** -0.5, 6
    total = [n + steps for n in lens]
    x = {name: wl.f32_to_bf16_bits(rng.standard_normal((B, max(total), h, d), dtype=np.float32)) for name, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    dev, host = {n: hp.dev_bf16(b) for n, b in x.items()}, {n: hp.widen(b) for n, b in x.items()}
    freq = tr._frequencies(d // 2)
    f = torch.from_numpy(freq).cuda()
    k_pages, v_pages = (torch.zeros(B * cols, page_rows, Hkv, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.from_numpy(rng.permutation(B * cols).astype(np.int32).reshape(B, cols)).cuda()
    rows = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = lib.paged_cache(k_pages, v_pages, table, rows)
    n = max(lens)
    place = torch.arange(n, dtype=torch.int32, device="cuda").expand(1, B, n)
    q_turned = torch.zeros(B, n, Hq, d, device="cuda", dtype=torch.bfloat16)
    prompt = {name: t[:, :n].contiguous() for name, t in dev.items()}
    lib.burst_attn_cache_append(lib.shape(B, Hq, Hkv, d, n, 0, 1.0), cache, prompt["k"], prompt["v"], rows, lib.rope(place, f), prompt["q"], q_turned)
    # the prompt's own attention, over the turned keys that the cache holds
    k_turned = torch.empty_like(prompt["k"])
    lib.burst_attn_rope(lib.shape(B, Hq, Hkv, d, n, 0, 1.0), lib.rope(place, f), prompt["q"], torch.empty_like(prompt["q"]), prompt["k"], k_turned)
    for b in range(B):
        page, r = (torch.from_numpy(a).cuda() for a in co.slots(table.cpu().numpy(), page_rows, b, np.arange(lens[b])))
        assert torch.equal(k_pages[page, r], k_turned[b, :lens[b]])
    # the captured token
    q1, k1, v1 = (torch.zeros(B, 1, h, d, device="cuda", dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    qt, o, lse = torch.zeros_like(q1), torch.zeros(B, 1, Hq, d, device="cuda"), torch.zeros(B, Hq, 1, device="cuda")
    at = torch.zeros(1, B, 1, dtype=torch.int32, device="cuda")
    shp, rope = lib.shape(B, Hq, Hkv, d, 1, cols * page_rows, scale), lib.rope(at, f)
    ws = torch.empty(lib.burst_attn_decode_workspace_bytes(shp), device="cuda", dtype=torch.uint8)

    def token(stream):
        lib.burst_attn_cache_append(shp, cache, k1, v1, None, rope, q1, qt, stream=stream)
        lib.burst_attn_decode(shp, cache, qt, o, lse, ws, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        token(torch.cuda.current_stream().cuda_stream)
    for s in range(steps):
        for name, t in (("q", q1), ("k", k1), ("v", v1)):
            for b in range(B):
                t[b, 0] = dev[name][b, lens[b] + s]
        at[0, :, 0] = rows
        rows += 1
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
        token(None)                                                        # eager, the same rows once more: the same bits
        torch.cuda.synchronize()
        assert np.array_equal(o.double().cpu().numpy(), got) and np.array_equal(lse.double().cpu().numpy(), got_lse)
        for b in range(B):
            m = lens[b] + s + 1
            p = np.arange(m)[None, None]
            kt = co.rope(host["k"][b:b + 1, :m], p, freq, [0] * (d // 2))
            kt = hp.widen(wl.f32_to_bf16_bits(kt.astype(np.float32)))
            qr = co.rope(host["q"][b:b + 1, m - 1:m], p[..., -1:], freq, [0] * (d // 2))
            qr = hp.widen(wl.f32_to_bf16_bits(qr.astype(np.float32)))
            O, L = oc.mha_attention_fwd(qr, kt, host["v"][b:b + 1, :m], scale)
            # turned numbers that fell on the other side of a rounding: up to a bf16 step in some elements, far inside the bar of the step
            assert np.abs(got[b] - O[0]).max() <= 2e-3 * np.abs(O).max() and np.abs(got_lse[b] - L[0]).max() <= hp.LSE_TOL


def test_shards_of_a_ring_joined(lib):
    """A cache dealt to four devices in stripes: each attends its own rows, burst_attn_lse_merge joins the results."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 86000))
    G, n, Hq, Hkv, d = 4, 1003, 8, 2, 128
    k, v = (wl.f32_to_bf16_bits(rng.standard_normal((1, n, Hkv, d), dtype=np.float32)) for _ in range(2))
    q, q_host = queries(rng, 1, Hq, d)
    o, lse = torch.zeros(1, 1, Hq, d, device="cuda"), torch.full((1, Hq, 1), -math.inf, device="cuda")
    for g in range(G):
        mine = np.arange(g, n, G)
        P = Paged(lib, rng, [mine.size], 16, Hkv, d)
        page, r = (torch.from_numpy(a).cuda() for a in co.slots(P.table, 16, 0, np.arange(mine.size)))
        P.dev["k"][page, r], P.dev["v"][page, r] = hp.dev_bf16(k)[0, mine], hp.dev_bf16(v)[0, mine]
        o_part, lse_part = run_decode(lib, P, q, 0.09, mine.size)
        lib.burst_attn_lse_merge(lib.shape(1, Hq, Hkv, d, 1, n, 0.09), o, lse, o_part, lse_part)
    O, L = oc.mha_attention_fwd(q_host[:, None], hp.widen(k), hp.widen(v), 0.09)
    assert np.abs(o.double().cpu().numpy() - O).max() <= 2e-5 * np.abs(O).max() + 1e-6
    assert np.abs(lse.double().cpu().numpy() - L).max() <= 1e-5


def test_keys_alone_are_turned_and_one_query_head_for_each(lib):
    """An append without queries; and the bits of one with them."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(11)
    k, v, q = (torch.randn(2, 7, 3, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(3))
    rope = lib.rope(torch.randint(0, 9999, (1, 2, 7), generator=gen, device="cuda", dtype=torch.int32), torch.from_numpy(tr._frequencies(32)).cuda())
    pages = []
    for with_q in (False, True):
        P = Paged(lib, np.random.Generator(np.random.PCG64(5)), [20, 7], 16, 3, 64)
        args = dict(q=q, q_out=torch.empty_like(q)) if with_q else {}
        lib.burst_attn_cache_append(lib.shape(2, 3, 3, 64, 7, 0, 1.0), P.cache, k, v, None, rope, **args)
        pages.append(P)
    assert all(torch.equal(pages[0].dev[x], pages[1].dev[x]) for x in "kv")


@pytest.mark.parametrize("Hq,Hkv,page_rows", [(130, 1, 1 << 12), (97, 97, 16), (512, 4, 80)])
def test_heads_and_pages_of_unusual_sizes(lib, Hq, Hkv, page_rows):
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 83300 + Hq))
    rows = [700, 0, 3]
    P = Paged(lib, rng, rows, page_rows, Hkv, 64, spare=1)
    q, q_host = queries(rng, 3, Hq, 64)
    o, lse = run_decode(lib, P, q, 0.125, 700, [3, 0, 1])
    check_decode(o, lse, P.decode(q_host, 0.125, [3, 0, 1]), 700, 64)
