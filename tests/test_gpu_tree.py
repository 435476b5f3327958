"""Attention of a few new tokens over a paged cache, on the GPU against the fp64 reference.

Tolerances, with u = 2^-24 and A the largest sum of |q| |K| of a token's head times the scale, as for one new token: a score is a sum of head_dim exact
products in fp32, off by at most head_dim u A, and its conversion to base 2 by 4 u A: e = (head_dim + 4) u A.  Lse is off by at most e, (n + 16) u for the
sum of n numbers, exponential and logarithm, and 4 u of its own size.  O, whose numbers P go in whole (to 2^-30 of each), by (2 e + (n + 16) u + 2^-30)
sum P |V|; in bf16 the result is rounded by half a step, 2^-8 of it, and with more than 32 columns (tokens times query heads of a key head) so is each P."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import helpers as hp
from tests import test_gpu_paged_cache as tp

pytestmark = pytest.mark.gpu


def random_tree(rng, n, reach=4):
    """Words of a random tree of n tokens: each sees its ancestors and itself."""
    words = []
    for i in range(n):
        parent = int(rng.integers(max(-1, i - reach), i)) if i else -1
        words.append((words[parent] if parent >= 0 else 0) | 1 << i)
    return words


def signed(words):
    return [w - (1 << 64) if w >> 63 else w for w in words]


def run_tree(lib, P, q, scale, max_rows, tokens=None, seen=None, first=None, sinks=0, elsewhere=False, o_type="f32", want_lse=True, ws=None):
    """seen: a list of lists of words, padded here; results over 7s."""
    import torch
    B, sq, Hq, d = q.shape
    shp = lib.shape(B, Hq, P.dev["k"].size(2), d, sq, max_rows, scale)
    o = torch.full((B, sq, Hq, d), 7.0, device="cuda", dtype=torch.float32 if o_type == "f32" else torch.bfloat16)
    lse = torch.full((B, Hq, sq), 7.0, device="cuda") if want_lse else None
    if ws is None:
        ws = torch.full((lib.burst_attn_tree_workspace_bytes(shp),), 255, device="cuda", dtype=torch.uint8)   # NaN everywhere
    t32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")
    words = None if seen is None else torch.tensor([signed(w) + [-1] * (sq - len(w)) for w in seen], dtype=torch.int64, device="cuda")
    tree = lib.tree(words, t32(first), t32(tokens), sinks, elsewhere)
    lib.burst_attn_tree(shp, P.cache, tree, q, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


def queries(rng, B, sq, Hq, d):
    bits = wl.f32_to_bf16_bits(rng.standard_normal((B, sq, Hq, d), dtype=np.float32))
    return hp.dev_bf16(bits), hp.widen(bits)


def check_tree(o, lse, ref, n, d, bf16=False, wide=False):
    O, lse_ref, weight, size = ref
    u = 2.0 ** -24
    e = (d + 4) * u * size                                                     # [batch, heads, tokens]
    got, there = o.double().cpu().numpy(), ~np.isnan(O)
    tol = (2 * np.moveaxis(e, 1, 2)[..., None] + (n + 16) * u + (2.0 ** -8 if bf16 and wide else 2.0 ** -30)) * weight
    if bf16:
        tol = tol + 2.0 ** -8 * np.maximum(np.abs(O) + tol, 2.0 ** -126)
    assert (np.abs(got - O) <= tol)[there].all(), float((np.abs(got - O) - tol)[there].max())
    assert (got[~there] == 7.0).all()                                          # padding stays as it was
    if lse is not None:
        l, there = lse.double().cpu().numpy(), ~np.isnan(lse_ref)
        dead = lse_ref == -np.inf
        assert (l[dead] == -np.inf).all() and (l[~there] == 7.0).all()
        assert (np.moveaxis(got, 1, 2)[dead] == 0).all()
        live = there & ~dead
        assert (np.abs(l - np.where(live, lse_ref, 0)) <= e + (n + 16) * u + 4 * u * np.abs(lse_ref))[live].all()


def reference(P, q_host, tokens, scale, **kw):
    return co.tree(q_host, P.host["k"], P.host["v"], P.table, P.rows, tokens, scale, k_scale=P.k_scale, v_scale=P.v_scale, **kw)


CASES = [
    # rows, tokens, sq, tree, page rows, q_heads, kv_heads, head_dim, e4m3, by head, type of O
    ([1], [1], 1, False, 16, 1, 1, 64, False, False, "f32"),
    ([777], [5], 5, False, 16, 12, 12, 64, False, False, "bf16"),
    ([5, 6, 64, 65, 130, 63], [5, 3, 5, 5, 1, 0], 5, True, 16, 8, 2, 128, False, False, "f32"),
    ([200, 64, 257, 7], [64, 64, 33, 7], 64, True, 16, 2, 2, 128, False, True, "f32"),
    ([300, 70], [16, 9], 16, True, 48, 16, 2, 128, False, False, "bf16"),         # 128 columns
    ([300, 70], [16, 9], 16, True, 48, 16, 2, 128, False, False, "f32"),
    ([513, 40], [40, 3], 40, True, 64, 32, 4, 64, False, False, "bf16"),          # 320 columns, a last block of 64
    ([1000, 3, 449], [7, 3, 0], 7, True, 1, 6, 2, 128, False, False, "f32"),
    ([333, 161], [11, 2], 11, True, 5, 9, 3, 64, False, False, "f32"),
    ([2000], [3], 3, True, 256, 17, 1, 128, False, False, "f32"),
    ([129, 700], [8, 6], 8, True, 16, 64, 8, 128, True, False, "bf16"),
    ([129, 700], [64, 6], 64, True, 7, 8, 1, 128, True, True, "f32"),
    ([99, 450], [12, 12], 12, True, 32, 5, 5, 64, True, False, "f32"),
    ([450, 31], [50, 31], 50, True, 24, 16, 4, 64, True, True, "bf16"),
    ([3000], [64], 64, True, 16, 4, 1, 64, False, False, "f32"),                  # dealt, 256 columns
]


@pytest.mark.parametrize("case", CASES)
def test_tree_against_the_reference(lib, case):
    rows, tokens, sq, is_tree, page_rows, Hq, Hkv, d, f8, by_head, o_type = case
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90000 + sum(rows) + Hq))
    P = tp.Paged(lib, rng, rows, page_rows, Hkv, d, f8, by_head)
    q, q_host = queries(rng, len(rows), sq, Hq, d)
    seen = [random_tree(rng, n) for n in tokens] if is_tree else None
    print(f"tree {case}", flush=True)
    ref = reference(P, q_host, tokens, d ** -0.5, seen=seen)
    for max_rows in sorted({max(rows), P.table.shape[1] * page_rows}):
        o, lse = run_tree(lib, P, q, d ** -0.5, max_rows, tokens, seen, o_type=o_type)
        check_tree(o, lse, ref, max(rows), d, o_type == "bf16", sq * Hq // Hkv > 32)
    o2, _ = run_tree(lib, P, q, d ** -0.5, max_rows, tokens, seen, o_type=o_type, want_lse=False)
    assert o.equal(o2)                                                         # the same call, the same bits, with Lse and without


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("sq,group", [(6, 4), (20, 8)])
def test_windows_and_first_rows(lib, sq, group, f8):
    """Windows that begin in different tiles for the tokens of a sequence, before its first row, behind its last; first rows that stay; either alone."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90100 + sq + f8))
    rows, d, Hkv = [400, 700, 150, 90, 1200], 128, 2
    tokens = [sq, sq, sq - 2, sq, 1]
    P = tp.Paged(lib, rng, rows, 16, Hkv, d, f8)
    q, q_host = queries(rng, 5, sq, Hkv * group, d)
    seen = [random_tree(rng, n) for n in tokens]
    first = rng.integers(-50, 1300, (5, sq))
    first[0] = 300 + np.arange(sq) * 10
    first[1] = 600
    first[2, 0], first[2, 1] = 2 ** 31 - 1, -2 ** 31
    for sinks in (0, 1, 4, 64, 100, 2 ** 31 - 1):
        for f in (first.tolist(), None):
            o, lse = run_tree(lib, P, q, 0.09, 1200, tokens, seen, f, sinks)
            check_tree(o, lse, reference(P, q_host, tokens, 0.09, seen=seen, first=f, sinks=sinks), 1200, d)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 1), (64, 6, 6)])
def test_words_of_any_kind(lib, d, Hq, Hkv):
    """Words that leave a token without rows (not even its own), that see later tokens, all, none; bits of tokens that are not there; nothing older."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90200 + d))
    sq, rows, tokens = 64, [64, 64, 40, 128, 10], [64, 64, 40, 64, 10]
    P = tp.Paged(lib, rng, rows, 16, Hkv, d)
    q, q_host = queries(rng, 5, sq, Hq, d)
    seen = [[int(x) for x in rng.integers(0, 2 ** 64, n, dtype=np.uint64)] for n in tokens]
    seen[0][3], seen[0][5], seen[0][63], seen[1][0] = 0, 2 ** 64 - 1, 1 << 63, 1 << 63
    seen[2] = [0] * 40
    seen[4] = [w & ~0x3ff for w in seen[4]]                                    # only bits of tokens that are not there
    o, lse = run_tree(lib, P, q, 0.1, 128, tokens, seen)
    ref = reference(P, q_host, tokens, 0.1, seen=seen)
    assert (ref[1][2, :, :40] == -np.inf).all() and (ref[1][4, :, :10] == -np.inf).all()
    check_tree(o, lse, ref, 128, d)


def test_more_tokens_than_rows_and_counts_out_of_range(lib):
    """tokens beyond sq or below 0, rows below tokens, beyond the table and below 0, and a bound that cuts off new rows."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90300))
    d, sq = 64, 6
    P = tp.Paged(lib, rng, [3, 60, 64, 64, 64], 16, 2, d, cols=4)
    P.rows = [3, 60, 10 ** 6, -5, 64]
    P.put_rows.copy_(torch.tensor(P.rows, dtype=torch.int32))
    tokens = [6, -2, 100, 4, 5]
    q, q_host = queries(rng, 5, sq, 4, d)
    seen = [random_tree(rng, sq) for _ in range(5)]
    for bound in (64, 61, 58, 2, 0):
        for w in (seen, None):
            o, lse = run_tree(lib, P, q, 0.1, bound, tokens, w)
            check_tree(o, lse, reference(P, q_host, tokens, 0.1, seen=w, max_rows=bound), 64, d)


@pytest.mark.parametrize("f8,page_rows", [(False, 16), (False, 6), (True, 32)])
@pytest.mark.parametrize("group", [2, 10])
def test_what_is_not_seen_may_hold_anything(lib, f8, page_rows, group):
    """NaN and infinities in every row that no token of any sequence sees: behind the last row, between the first rows and the windows, drafts
    that nobody sees, spare pages."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90400 + page_rows))
    rows, tokens, sq, d, sinks = [100, 37, 300, 161], [9, 3, 13, 0], 13, 64, 5
    P = tp.Paged(lib, rng, rows, page_rows, 2, d, f8)
    first = [[33] * sq, [0] * sq, [200 + i for i in range(sq)], [150] * sq]
    seen = [[w & ~0b101 for w in random_tree(rng, n)] for n in tokens]         # new tokens 0 and 2 are seen by none
    visible = np.zeros((P.n_pages, page_rows), bool)
    for b in range(4):
        vis = co.tree_visible(tokens[b], rows[b], rows[b], seen[b], first[b], sinks).any(0)
        page, r = co.slots(P.table, page_rows, b, np.flatnonzero(vis))
        visible[page, r] = True
    hidden = torch.from_numpy(~visible).cuda()
    for name, bad in (("k", float("nan")), ("v", float("nan") if f8 else float("inf"))):
        P.dev[name].view(torch.uint8 if f8 else torch.bfloat16)[hidden] = 0x7f if f8 else bad
    q, q_host = queries(rng, 4, sq, 2 * group, d)
    o, lse = run_tree(lib, P, q, 0.125, 300, tokens, seen, first, sinks)
    check_tree(o, lse, reference(P, q_host, tokens, 0.125, seen=seen, first=first, sinks=sinks), 300, d)


@pytest.mark.parametrize("page_rows", [16, 5])
def test_pages_that_are_none(lib, page_rows):
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90500 + page_rows))
    rows, tokens = [200, 200, 170], [4, 4, 4]
    P = tp.Paged(lib, rng, rows, page_rows, 2, 128)
    P.table[0, 3], P.table[1, :] = P.n_pages, -1
    P.table[2, 0], P.table[2, (170 - 1) // page_rows] = 2 ** 31 - 1, -2 ** 31  # (the last: of new rows)
    P.put_table.copy_(torch.from_numpy(P.table))
    q, q_host = queries(rng, 3, 4, 4, 128)
    o, lse = run_tree(lib, P, q, 0.09, 200, tokens)
    ref = reference(P, q_host, tokens, 0.09)
    assert (ref[1][1] == -np.inf).all()
    check_tree(o, lse, ref, 200, 128)


def test_infinities_and_nan_that_are_seen(lib):
    """A NaN key makes NaN of its heads' results for the tokens that see it, and of no other sequence's or head's; a value's infinity is its element's."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90600))
    P = tp.Paged(lib, rng, [300, 300], 16, 3, 64)
    q, q_host = queries(rng, 2, 4, 6, 64)
    page, r = co.slots(P.table, 16, 0, 123)
    P.dev["k"][page, r, 0, 5] = float("nan")
    P.dev["v"][page, r, 1, 7] = float("inf")
    for o_type in ("f32", "bf16"):
        o, lse = run_tree(lib, P, q, 0.125, 300, o_type=o_type)
        assert torch.isnan(o[0, :, :2]).all() and torch.isnan(lse[0, :2]).all()
        assert (o[0, :, 2:4, 7] == math.inf).all() and torch.isfinite(o[0, :, 2:4, :7]).all() and torch.isfinite(lse[0, 2:4]).all()
        assert torch.isfinite(o[0, :, 4:]).all() and torch.isfinite(o[1]).all() and torch.isfinite(lse[1]).all()


def test_scores_of_all_sizes(lib):
    """Scores that grow from row to row, that fall, and far below zero: the running maximum follows; nothing overflows or vanishes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90700))
    P = tp.Paged(lib, rng, [1000] * 4, 16, 1, 64, fill=0.0)
    ramp = np.linspace(-600.0, 600.0, 1000)
    for b, s in enumerate((ramp, ramp[::-1], np.full(1000, -700.0), np.where(np.arange(1000) == 517, 900.0, -900.0))):
        page, r = co.slots(P.table, 16, b, np.arange(1000))
        P.dev["k"][page, r, 0, 0] = torch.from_numpy(s.copy()).to(torch.bfloat16).cuda()
        P.dev["v"][page, r, 0] = torch.randn(1000, 64, device="cuda").to(torch.bfloat16)
    P.refresh()
    for sq in (3, 40):
        q = torch.zeros(4, sq, 2, 64, device="cuda", dtype=torch.bfloat16)
        q[:, :, 0, 0], q[:, :, 1, 0] = 1.0, -1.0
        q[:, 1] *= 0.5
        o, lse = run_tree(lib, P, q, 1.0, 1000)
        check_tree(o, lse, reference(P, q.double().cpu().numpy(), [sq] * 4, 1.0), 1000, 64)


def test_elsewhere_and_joined(lib):
    """A cache in two halves, the new tokens' rows in the second: each half's results joined are those over the whole."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90800))
    sq, d, Hq, Hkv, rows, tokens = 7, 64, 8, 2, [500, 77], [7, 7]
    P = tp.Paged(lib, rng, rows, 16, Hkv, d)
    q, q_host = queries(rng, 2, sq, Hq, d)
    seen = [random_tree(rng, n) for n in tokens]
    half = [160, 32]                                                          # (multiples of the page)
    one, two = (tp.Paged.__new__(tp.Paged) for _ in range(2))
    for X, table, n in ((one, P.table, half), (two, np.stack([np.roll(P.table[b], -h // 16) for b, h in enumerate(half)]), [r - h for r, h in zip(rows, half)])):
        X.dev = P.dev
        X.cache = lib.paged_cache(P.dev["k"], P.dev["v"], torch.from_numpy(np.ascontiguousarray(table)).cuda(), torch.tensor(n, dtype=torch.int32, device="cuda"))
    acc, lse_acc = torch.zeros(2, sq, Hq, d, device="cuda"), torch.full((2, Hq, sq), -math.inf, device="cuda")
    for X, away in ((one, True), (two, False)):
        o, lse = run_tree(lib, X, q, 0.125, 512, tokens, seen, elsewhere=away)
        lib.burst_attn_lse_merge(lib.shape(2, Hq, Hkv, d, sq, 0, 0.125), acc, lse_acc, o, lse)
    O, L, weight, size = reference(P, q_host, tokens, 0.125, seen=seen)
    assert np.abs(acc.double().cpu().numpy() - O).max() <= 1e-5 and np.abs(lse_acc.double().cpu().numpy() - L).max() <= 1e-5


@pytest.mark.parametrize("d", [64, 128])
def test_one_token_as_the_call_for_one(lib, d):
    """sq = 1: what burst_attn_decode gives, to the order of fp32 sums."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90900 + d))
    rows = [1500, 3, 0, 64, 700]
    P = tp.Paged(lib, rng, rows, 16, 2, d)
    q, q_host = queries(rng, 5, 1, 8, d)
    o, lse = run_tree(lib, P, q, 0.1, 1500, [1, 1, 1, 1, 1])
    o1, lse1 = tp.run_decode(lib, P, q, 0.1, 1500)
    some = [0, 1, 3, 4]
    assert (o - o1).abs().max() <= 2.0 ** -18 and (lse - lse1)[some].abs().max() <= 2.0 ** -18
    assert (o[2] == 0).all() and (lse[2] == -math.inf).all()


@pytest.mark.parametrize("B", [1, 63, 64, 65, 130, 300])
@pytest.mark.parametrize("group", [1, 9])
def test_scan_over_the_sequences(lib, B, group):
    """Batches around the size at which the scan changes, some sequences without tokens, one long: sampled ones against the reference."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91000 + B))
    rows = rng.integers(8, 200, B).tolist()
    tokens = rng.integers(0, 9, B).tolist()
    rows[B // 2], tokens[B // 2] = 4000, 8
    P = tp.Paged(lib, rng, [2000], 16, 1, 64)
    P.rows, P.table = rows, rng.integers(0, P.n_pages, (B, 250)).astype(np.int32)
    P.cache = lib.paged_cache(P.dev["k"], P.dev["v"], torch.from_numpy(P.table).cuda(), torch.tensor(rows, dtype=torch.int32, device="cuda"))
    q, q_host = queries(rng, B, 8, group, 64)
    o, lse = run_tree(lib, P, q, 0.125, 4000, tokens)
    some = sorted({0, B // 2, B - 1, B // 3, min(B - 1, 63), min(B - 1, 64)})
    O, L, w, s = co.tree(q_host[some], P.host["k"], P.host["v"], P.table[some], [rows[b] for b in some], [tokens[b] for b in some], 0.125)
    check_tree(o[some], lse[some], (O, L, w, s), 4000, 64)


def test_every_way_of_dealing(lib):
    """Direct and dealt, 16 to 128 columns, blocks that only longer sequences have, by burst_attn_tree_plan."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91100))
    for B, Hkv, sq, Hq, longest, columns, direct in ((3, 2, 8, 8, 1500, 32, False), (3, 2, 8, 8, 100, 32, True), (3, 2, 4, 8, 1500, 16, False), (3, 2, 3, 8, 300, 16, True), (3, 2, 16, 8, 1500, 64, False), (3, 2, 16, 8, 200, 64, True),
                                                     (2, 2, 30, 8, 1500, 128, False), (2, 2, 40, 8, 1500, 128, False), (70, 8, 20, 8, 3000, 32, True), (70, 8, 2, 8, 3000, 16, True), (70, 8, 50, 8, 900, 64, True),
                                                     (130, 4, 30, 16, 300, 128, True), (70, 4, 64, 16, 300, 128, True)):
        assert lib.burst_attn_tree_plan(lib.shape(B, Hq, Hkv, 64, sq, longest, 1.0))[1:] == (columns, direct)
        rows = rng.integers(sq, longest, B).tolist()
        rows[0] = longest
        tokens = rng.integers(0, sq + 1, B).tolist()
        tokens[0] = sq
        P = tp.Paged(lib, rng, rows, 16, Hkv, 64)
        q, q_host = queries(rng, B, sq, Hq, 64)
        print("tree plan", B, Hkv, sq, Hq, longest, flush=True)
        o, lse = run_tree(lib, P, q, 0.125, longest, tokens)
        some = [0, 1, B - 1]
        ref = co.tree(q_host[some], P.host["k"], P.host["v"], P.table[some], [rows[b] for b in some], [tokens[b] for b in some], 0.125)
        check_tree(o[some], lse[some], ref, longest, 64)


def test_strided_views_and_one_tree_for_all(lib):
    """q, o and lse as parts of larger tensors whose rest stays as it is; one tree, one list of first rows and one row of the table for all."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91200))
    B, sq, Hq, Hkv, d, rows = 3, 5, 6, 2, 128, [300, 200, 250]
    P = tp.Paged(lib, rng, [300, 300, 300], 16, Hkv, d)
    P.rows, P.table = rows, np.repeat(P.table[:1], B, 0)
    words = random_tree(rng, sq)
    one_table = torch.from_numpy(P.table[:1].copy()).cuda().expand(B, -1)
    cache = lib.paged_cache(P.dev["k"], P.dev["v"], one_table, torch.tensor(rows, dtype=torch.int32, device="cuda"))
    tree = lib.tree(torch.tensor([words], device="cuda").expand(B, -1), torch.tensor([[100 + i for i in range(sq)]], dtype=torch.int32, device="cuda").expand(B, -1))
    q, q_host = queries(rng, B, sq, Hq, d)
    wide_q = torch.full((B, sq + 2, Hq + 5, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide_q[:, 1:1 + sq, 2:2 + Hq] = q
    wide_o, wide_lse = torch.full((B, sq + 2, Hq + 3, d), 7.0, device="cuda"), torch.full((B, Hq + 1, sq + 4), 7.0, device="cuda")
    shp = lib.shape(B, Hq, Hkv, d, sq, 300, 0.09)
    ws = torch.empty(lib.burst_attn_tree_workspace_bytes(shp) + 256, device="cuda", dtype=torch.uint8)
    lib.burst_attn_tree(shp, cache, tree, wide_q[:, 1:1 + sq, 2:2 + Hq], wide_o[:, :sq, 1:1 + Hq], wide_lse[:, :Hq, 3:3 + sq], ws)
    torch.cuda.synchronize()
    ref = co.tree(q_host, P.host["k"], P.host["v"], P.table, rows, [sq] * B, 0.09, seen=[words] * B, first=[[100 + i for i in range(sq)]] * B)
    check_tree(wide_o[:, :sq, 1:1 + Hq], wide_lse[:, :Hq, 3:3 + sq], ref, 300, d)
    assert (wide_o[:, sq:] == 7).all() and (wide_o[:, :, 0] == 7).all() and (wide_o[:, :, Hq + 1:] == 7).all()
    assert (wide_lse[:, Hq:] == 7).all() and (wide_lse[:, :, :3] == 7).all() and (wide_lse[:, :, 3 + sq:] == 7).all()


def test_two_graphs_one_workspace(lib):
    """Two captured calls that share a workspace, replayed in turn with eager calls, other lengths, trees and windows between: the eager results."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91300))
    B, Hkv, sq, longest = 5, 3, 6, 3000
    P = tp.Paged(lib, rng, [longest] * B, 16, Hkv, 64)
    shp = lib.shape(B, Hkv * 4, Hkv, 64, sq, longest, 0.125)
    assert not lib.burst_attn_tree_plan(shp)[2]
    ws = torch.full((lib.burst_attn_tree_workspace_bytes(shp),), 255, device="cuda", dtype=torch.uint8)
    q = [queries(rng, B, sq, Hkv * 4, 64)[0] for _ in range(2)]
    o = [torch.zeros(B, sq, Hkv * 4, 64, device="cuda") for _ in range(2)]
    lse = [torch.zeros(B, Hkv * 4, sq, device="cuda") for _ in range(2)]
    first, tokens = torch.zeros(B, sq, dtype=torch.int32, device="cuda"), torch.full((B,), sq, dtype=torch.int32, device="cuda")
    seen = torch.zeros(B, sq, dtype=torch.int64, device="cuda")
    tree = lib.tree(seen, first, tokens, 3)
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            lib.burst_attn_tree(shp, P.cache, tree, q[i], o[i], lse[i], ws)
    for turn in range(4):
        P.put_rows.copy_(torch.tensor(rng.integers(sq, longest, B), dtype=torch.int32))
        tokens.copy_(torch.tensor(rng.integers(0, sq + 1, B), dtype=torch.int32))
        seen.copy_(torch.tensor(rng.integers(0, 64, (B, sq))))
        first.copy_((P.put_rows * 0.3).to(torch.int32)[:, None].expand(-1, sq) * (turn % 2))
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        got = [(a.clone(), b.clone()) for a, b in zip(o, lse)]
        for i in range(2):
            lib.burst_attn_tree(shp, P.cache, tree, q[i], o[i], lse[i], ws)
            torch.cuda.synchronize()
            assert torch.equal(o[i], got[i][0]) and torch.equal(lse[i], got[i][1])


def test_streams_of_their_own(lib):
    """Calls on two streams at once, each with its workspace, against the calls one after the other."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91400))
    P = tp.Paged(lib, rng, [2000, 900], 16, 2, 128)
    q = [queries(rng, 2, 9, 16, 128)[0] for _ in range(2)]
    want = [run_tree(lib, P, x, 0.09, 2000) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    shp, tree = lib.shape(2, 16, 2, 128, 9, 2000, 0.09), lib.tree()
    ws = [torch.empty(lib.burst_attn_tree_workspace_bytes(shp), device="cuda", dtype=torch.uint8) for _ in range(2)]
    got = [(torch.empty_like(o), torch.empty_like(l)) for o, l in want]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, s in enumerate(streams):
            lib.burst_attn_tree(shp, P.cache, tree, q[i], *got[i], ws[i], stream=s.cuda_stream)
    torch.cuda.synchronize()
    for (o, l), (o2, l2) in zip(want, got):
        assert torch.equal(o, o2) and torch.equal(l, l2)


def test_more_sequences_than_a_launch_has_threads_for(lib):
    """2^24 sequences and some of more than a tile, which in work-groups of four waves would be 2^32 threads: as many rows, the same result."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91700))
    B, d, longest, some = (1 << 24) + 100, 64, 150, 128
    P = tp.Paged(lib, rng, [longest], 160, 1, d)
    table = torch.from_numpy(P.table.astype(np.int32)).cuda().expand(B, -1)
    lengths = torch.arange(B, device="cuda", dtype=torch.int32) % some + (longest - some + 1)
    cache = lib.paged_cache(P.dev["k"], P.dev["v"], table, lengths)
    q, q_host = queries(rng, 1, 1, 1, d)
    shp = lib.shape(B, 1, 1, d, 1, longest, 0.125)
    assert lib.burst_attn_tree_plan(shp) == (B, 16, True) and lib.burst_attn_tree_workspace_bytes(shp) == 0
    o = torch.full((B, 1, 1, d), 7.0, device="cuda", dtype=torch.bfloat16)
    lib.burst_attn_tree(shp, cache, lib.tree(), q.expand(B, -1, -1, -1), o)
    torch.cuda.synchronize()
    rows = lengths[:some].tolist()
    ref = co.tree(np.repeat(q_host, some, 0), P.host["k"], P.host["v"], np.repeat(P.table, some, 0), rows, [1] * some, 0.125)
    check_tree(o[:some], None, ref, longest, d, bf16=True)
    assert torch.equal(o[some:].view(torch.int16), o[:-some].view(torch.int16))


def test_offsets_beyond_32_bits(lib):
    """Pages 1 GiB and heads 4 GiB from each other."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91500))
    head, d = 1 << 31, 128                                                    # (elements)
    flat = torch.empty(2 * head, device="cuda", dtype=torch.bfloat16)
    x = flat.as_strided((4, 64, 2, d), (1 << 29, d, head, 1))[1:4]
    v = flat[64 * 128:].as_strided((4, 64, 2, d), (1 << 29, d, head, 1))[1:4]
    k_host, v_host = (torch.empty(3, 64, 2, d).normal_(generator=torch.Generator().manual_seed(i)).to(torch.bfloat16) for i in (1, 2))
    x.copy_(k_host)
    v.copy_(v_host)
    table, rows = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda"), torch.tensor([150], dtype=torch.int32, device="cuda")
    cache = lib.paged_cache(x, v, table, rows)
    wide = lambda t: t.float().numpy().astype(np.float64)
    for sq in (3, 40):
        q, q_host = queries(rng, 1, sq, 4, d)
        o, lse = torch.full((1, sq, 4, d), 7.0, device="cuda"), torch.full((1, 4, sq), 7.0, device="cuda")
        shp = lib.shape(1, 4, 2, d, sq, 192, 0.09)
        ws = torch.empty(lib.burst_attn_tree_workspace_bytes(shp), device="cuda", dtype=torch.uint8)
        lib.burst_attn_tree(shp, cache, lib.tree(), q, o, lse, ws)
        check_tree(o, lse, co.tree(q_host, wide(k_host), wide(v_host), table.cpu().numpy(), [150], [sq], 0.09), 150, d)


def test_a_token_does_not_depend_on_its_batch(lib):
    """The same sequence alone and among others, the same tokens alone and with others behind them: other roundings in fp32 alone."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91600))
    rows = [1777, 50, 900, 3100]
    P = tp.Paged(lib, rng, rows, 16, 2, 128)
    q, _ = queries(rng, 4, 30, 8, 128)
    o, lse = run_tree(lib, P, q, 0.09, 3100)
    P.cache = lib.paged_cache(P.dev["k"], P.dev["v"], P.put_table[:1], P.put_rows[:1])
    o1, lse1 = run_tree(lib, P, q[:1], 0.09, 1777)
    assert (o1[0] - o[0]).abs().max() <= 2.0 ** -19 * o[0].abs().max() and (lse1[0] - lse[0]).abs().max() <= 2.0 ** -19
