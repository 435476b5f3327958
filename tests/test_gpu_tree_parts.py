"""What the weights of a drafted token's attention lose to the matrix products, on the GPU: O in bf16 is O in fp32, cast, but for 2^-16 of each weight, however many columns
(tokens times query heads of a key head) there are.

Tolerances, with u = 2^-24, n rows and W the sum of P |V| in 64 bits: both calls form the same scores and the same 24 bits of P, as the running maximum is a whole number.  Either sums n
products and n weights in fp32, in an order of its own, and divides: 2 (n + 16) u W each.  With more than 32 columns and O in bf16 each P is taken to 2^-16: 2^-16 W.  The cast is half
a step, 2^-8 of the result."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import test_gpu_paged_cache as tp
from tests.test_gpu_tree import queries, random_tree, run_tree

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def check_cast(o16, o32, weight, n):
    f, got, there = o32.double().cpu().numpy(), o16.double().cpu().numpy(), ~np.isnan(weight)
    t = (2.0 ** -16 + 4 * (n + 16) * U) * np.where(there, weight, 0)
    tol = t + 2.0 ** -8 * np.maximum(np.abs(f) + t, 2.0 ** -126)
    assert (np.abs(got - f) <= tol)[there].all(), (float((np.abs(got - f) - tol)[there].max()), int((np.abs(got - f) > tol)[there].sum()))


CASES = [
    # rows, tokens, sq, page rows, q_heads, kv_heads, head_dim, e4m3; the bound of the rows (a long one: dealt)
    ([40, 70], [9, 9], 9, 16, 8, 2, 128, False, 70),                # 36 columns
    ([40, 70], [9, 4], 9, 16, 8, 2, 128, False, 4096),
    ([55, 130], [12, 12], 12, 5, 16, 2, 128, False, 130),           # 96
    ([33, 61], [20, 17], 20, 16, 16, 2, 64, False, 8192),           # 160
    ([64, 90], [33, 20], 33, 7, 4, 2, 64, False, 90),               # 66
    ([40, 70], [9, 9], 9, 16, 8, 2, 128, True, 70),
    ([40, 70, 64], [40, 3, 64], 64, 16, 4, 1, 128, True, 4096),     # 256
    ([50, 20], [50, 20], 50, 24, 4, 4, 64, True, 50),
    ([40, 70], [8, 8], 8, 16, 8, 2, 128, False, 70),                # 32
    ([77, 300], [3, 3], 3, 16, 8, 2, 64, True, 4096),
]


@pytest.mark.parametrize("case", CASES)
def test_the_type_of_o_is_a_cast(lib, case):
    rows, tokens, sq, page_rows, Hq, Hkv, d, f8, bound = case
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 95000 + sum(rows) + Hq + d))
    P = tp.Paged(lib, rng, rows, page_rows, Hkv, d, f8, cols=-(-bound // page_rows))
    q, q_host = queries(rng, len(rows), sq, Hq, d)
    seen = [random_tree(rng, n) for n in tokens]
    scale = 0.25 * d ** -0.5
    print(f"parts {case}", flush=True)
    weight = co.tree(q_host, P.host["k"], P.host["v"], P.table, P.rows, tokens, scale, seen=seen, k_scale=P.k_scale, v_scale=P.v_scale)[2]
    o32, lse32 = run_tree(lib, P, q, scale, bound, tokens, seen)
    o16, lse16 = run_tree(lib, P, q, scale, bound, tokens, seen, o_type="bf16")
    check_cast(o16, o32, weight, max(rows))
    assert (lse16 - lse32).abs().max() <= 2 * (max(rows) + 16) * U + 8 * U * lse32.abs().max()      # (of the whole weights, either way)


@pytest.mark.parametrize("f8", [False, True])
def test_one_more_token_changes_nothing_but_roundings(lib, f8):
    """8 tokens over 4 query heads a key head are 32 columns, 9 are more than 32: the first 8 tokens' results agree, in bf16 too."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 95100 + f8))
    rows, sq, d, Hq, Hkv, scale = [59, 93, 41], 9, 128, 8, 2, 0.02
    P = tp.Paged(lib, rng, rows, 16, Hkv, d, f8)
    q, q_host = queries(rng, 3, sq, Hq, d)
    seen = [random_tree(rng, sq) for _ in rows]
    weight = co.tree(q_host, P.host["k"], P.host["v"], P.table, P.rows, [sq] * 3, scale, seen=seen, k_scale=P.k_scale, v_scale=P.v_scale)[2][:, :8]
    o32, _ = run_tree(lib, P, q, scale, 93, [sq] * 3, seen)
    o16, _ = run_tree(lib, P, q, scale, 93, [sq] * 3, seen, o_type="bf16")
    # the same eight tokens by themselves: the ninth one's row, which none of them sees, is the last
    P.rows = [r - 1 for r in rows]
    P.put_rows.copy_(torch.tensor(P.rows, dtype=torch.int32))
    few = [w[:8] for w in seen]
    o32_few, _ = run_tree(lib, P, q[:, :8].contiguous(), scale, 93, [8] * 3, few)
    o16_few, _ = run_tree(lib, P, q[:, :8].contiguous(), scale, 93, [8] * 3, few, o_type="bf16")
    assert np.abs((o32[:, :8] - o32_few).double().cpu().numpy()).max() <= 4 * (93 + 16) * U * weight.max()
    for o in (o16[:, :8], o16_few):
        check_cast(o, o32_few, weight, 93)


def test_infinities_of_many_columns(lib):
    """An infinity among the values is its element's for every token and head that sees it, whatever its weight rounds to, with O in bf16 as well."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 95200))
    P = tp.Paged(lib, rng, [300, 300], 16, 3, 64)
    page, r = co.slots(P.table, 16, 0, 123)
    P.dev["v"][page, r, 1, 7] = math.inf
    for sq in (12, 40):
        q, _ = queries(rng, 2, sq, 12, 64)
        for o_type in ("f32", "bf16"):
            o, lse = run_tree(lib, P, q, 0.125, 300, o_type=o_type)
            assert (o[0, :, 4:8, 7] == math.inf).all() and torch.isfinite(o[0, :, 4:8, :7]).all() and torch.isfinite(o[0, :, :4]).all() and torch.isfinite(o[0, :, 8:]).all()
            assert torch.isfinite(o[1]).all() and torch.isfinite(lse).all()
