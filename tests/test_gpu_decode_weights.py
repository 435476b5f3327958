"""How exactly the weights of one new token's attention go into the product with the values: all 24 bits of them.

Tolerance of the weights, with u = 2^-24.  Row t's score is one exact product (a query with a single 1, a key of bf16 or e4m3): S_t = scale * K_t,
scale a power of two.  Its size in base 2, x, is off by 5 u |x| (log2 e as a constant, its products with the scale and the key's scale, the product
with the score, one to spare), and its distance from the maximum is rounded once, by u (2 |x| + 1); so exp2 of it is off by ln 2 of these, and by
its own 2 u.  The values are 1 in one element of a row, 0 otherwise, so that O has each weight by itself, over a sum which all share:
O_t / O_0, with row 0's score 0, is off by the above, twice exp2's error for row 0 and the waves' rescaling by a power of two, and a rounding for the
product with 1 / sum on either side.  All scores are within 2, |x| within 3: ln 2 * (15 + 7) + 2 + 4 + 2 < 24 u."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import test_gpu_decode_values as tv
from tests import test_gpu_paged_cache as tp

U = 2.0 ** -24
WEIGHT_TOL = 24 * U


def _weights(rng, n, d, f8):
    """Scores S_0 = 0 and others within 2 that keys of the cache's type can have: (keys, the rows' scores over scale 1)."""
    x = rng.uniform(-2.0, 2.0, n)
    x[0] = 0.0
    if f8:      # multiples of 1 / 8 up to 2: numbers of e4m3 (over a scale of 2^-3: whole numbers up to 16)
        return np.round(8.0 * x), np.round(8.0 * x) / 8.0
    bits = wl.f32_to_bf16_bits(x.astype(np.float32))
    x = wl.bf16_bits_to_f64(bits)
    return x, x


def _split_error(weights, parts):
    """The largest relative error of weights (24 bits) cut into `parts` truncated bf16 numbers."""
    left = np.asarray(weights, np.float32)
    for _ in range(parts):
        left = left - (left.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    return float((left / np.asarray(weights, np.float32)).max())


@pytest.mark.parametrize("f8", [False, True])
def test_a_missing_part_would_show(f8):
    """On the CPU: the weights of the test below in two parts are further off than it allows; in three they are exact."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90100 + f8))
    _, s = _weights(rng, 64, 64, f8)
    w = np.exp(s - math.ceil(s.max() / math.log(2.0)) * math.log(2.0)).astype(np.float32)
    assert _split_error(w, 2) > 2 * WEIGHT_TOL and _split_error(w, 3) == 0.0


@pytest.mark.gpu
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", list(tv.MODES))
def test_weights_have_all_their_bits(lib, mode, d, f8):
    """The weights of 64 rows, one by one, against exp in 64 bits."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90100 + f8))
    Hkv, page_rows, n = tv.MODES[mode][0], 16, 64
    bound = tv.bound_of(mode, page_rows)
    rows = {"direct": [490], "dealt": [4000], "beside": [6000]}[mode]
    P = tp.Paged(lib, rng, rows, page_rows, Hkv, d, f8, cols=bound // page_rows, fill=0.0)
    at = np.sort(rng.permutation(rows[0])[:n])                              # the rows that have a weight to look at
    keys, s = _weights(np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90100 + f8)), n, d, f8)
    page, r = (torch.from_numpy(a).cuda() for a in co.slots(P.table, page_rows, 0, at))
    k, v = torch.zeros(n, Hkv, d), torch.zeros(n, Hkv, d)
    k[:, :, 7] = torch.from_numpy(keys).float()[:, None]
    v[torch.arange(n), :, torch.arange(n)] = 1.0
    bits = (lambda t: t.view(torch.uint8)) if f8 else lambda t: t
    for name, x in (("k", k), ("v", v)):
        bits(P.dev[name])[page, r] = bits(x.to(P.dev[name].dtype).cuda())
    if f8:
        P.cache._tensors[4].fill_(0.125)                                    # the keys' scales
        P.cache._tensors[5].fill_(0.75)
    q = torch.zeros(1, 1, 2 * Hkv, d, device="cuda", dtype=torch.bfloat16)
    q[..., 7] = 1.0
    shares, heads, direct = lib.burst_attn_decode_plan(lib.shape(1, 2 * Hkv, Hkv, d, 1, bound, 1.0), P.cache)
    assert direct == (mode == "direct") and (heads > 1) == (mode == "beside")
    print(f"weights, {mode} d={d} f8={f8}", flush=True)
    o, _ = tp.run_decode(lib, P, q, 1.0, bound)
    got = o[0, 0, :, :n].double().cpu().numpy()
    off = np.abs(got / got[:, :1] / np.exp(s) - 1.0)
    print("largest error %.1f u" % (off.max() / U), flush=True)
    assert (off <= WEIGHT_TOL).all()
