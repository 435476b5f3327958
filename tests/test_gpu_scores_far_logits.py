"""Scores and their gradient where logits are large finite numbers, on the GPU against the fp64 reference: words that are forbidden by -1e10, -1e30 or the type's lowest number, rows that
hold nothing else, rows far from zero.

Everything but Lse depends on differences alone, so the reference takes the logits minus their row's largest, in 64 bits (at -1e30 a Lse in 64 bits itself would say nothing of log v).

Tolerances, with u = 2^-24 and D the largest scale * |x - max| of a row's words that have a share (2^-160 and more): an exponent is a difference and a product with a number of two
roundings, 4 u D; the sum of v exponentials is off by (v + 8) u of itself and 4 u D; so log l by e = 4 u D + (v + 8) u + 2 u log v.  logp = scale (x - max) - log l: e and three roundings
of its own size.  Lse = scale max + log l: e and two roundings of its size and of scale max.  The entropy is a sum of p |log p| with these errors, log l - w / l: (2 (v + 8) u + 8 u D)
(1 + log v + entropy).  A gradient is scale times sums of products with p, which is off by 4 u D + (v + 8) u of itself where |Lse| is above 4096, and else also by the rounding of Lse and of
what is subtracted from it: 4 u (|Lse| + D + |log p|); and p below 2^-126, where an exponential may come out as 0, by that much whatever its size; half a step of
its type."""
import math

import numpy as np
import pytest

from oracle import lm_head_oracle as lmo
from paper_2509_19836_amd import workloads as wl
from tests.test_gpu_scores import run

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LARGEST = float(np.finfo(np.float32).max)


def lowest(dtype):
    import torch
    return torch.finfo(dtype).min


def rows_of(rng, v, dtype):
    """Rows at finite numbers far away, ordinary words beside such ones, differences of a few units far from zero."""
    import torch
    low, one = lowest(dtype), rng.standard_normal(v) * 3

    def beside(fill, share):
        row = np.where(rng.random(v) < share, one, fill)
        row[v // 2] = 0.25
        return row
    rows = [np.full(v, x) for x in (-1e10, -1e30, low, 1e10, 3e9, -low)]
    rows += [beside(x, s) for x in (-1e4, -1e9, -1e10, -1e30, low) for s in (0.5, 0.01)]
    rows += [-1e30 * rng.random(v), 1e30 * rng.random(v), np.where(rng.random(v) < 0.5, -1e10, low), np.where(rng.random(v) < 0.5, -np.inf, -1e10), 3e4 + 256 * rng.integers(0, 2, v)]
    rows.append(1e6 + rng.integers(0, 64, v) / 16 if dtype == torch.float32 else 4096 + 32.0 * rng.integers(0, 2, v))
    rows.append(np.where(np.arange(v) == v // 3, 5.0, low))
    return np.stack(rows)


def reference(x, y, n_top, scale):
    """logp, entropy, top_logp and log l from x - max, the words' order from x, Lse as an fp32 number has it."""
    top = x.max(1)
    ref = lmo.scores(x - top[:, None], y, n_top, scale)
    ref["top_ids"] = lmo.scores(x, y, n_top, scale)["top_ids"]
    every = lmo.scores(x - top[:, None], None, 0, scale)["lse"]
    logp = (x - top[:, None]) * scale - every[:, None]
    ref["top_logp"] = np.take_along_axis(logp, ref["top_ids"], 1)
    ref["log_l"], ref["lse"] = every, top * scale + every
    return ref


def spread(x, scale):
    d = scale * (x.max(1, keepdims=True) - x)
    return np.where(d < 160 * math.log(2), d, 0).max(1)


def near(a, b, tol, what):
    b = np.where(np.abs(b) > LARGEST, np.copysign(np.inf, b), b)
    with np.errstate(invalid="ignore"):
        same = (a == b) | (np.abs(a - b) <= tol)
    assert same.all(), (what, np.argwhere(~same)[:5].tolist(), a[~same][:5], b[~same][:5])


def check_scores(got, ref, x, scale):
    v, D = x.shape[1], spread(x, scale)
    e = 4 * U * D + (v + 8) * U + 2 * U * math.log(v)
    near(got["lse"], ref["lse"], e + 2 * U * np.abs(ref["lse"]) + 2 * U * scale * np.abs(x.max(1)), "lse")
    near(got["logp"], ref["logp"], e + 3 * U * np.abs(ref["logp"]), "logp")
    near(got["entropy"], ref["entropy"], (2 * (v + 8) * U + 8 * U * D) * (1 + math.log(v) + ref["entropy"]), "entropy")
    near(got["top_logp"], ref["top_logp"], e[:, None] + 3 * U * np.abs(ref["top_logp"]), "top_logp")
    assert np.array_equal(got["top_ids"], ref["top_ids"])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n,v", [(24, 300), (2112, 130), (24, 5003), (24, 70000), (24, 110000)])   # a wave a row (twice), four, sixteen, several work-groups
def test_scores(lib, n, v, kind):
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 96000 + v))
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    few = torch.from_numpy(rows_of(rng, v, dtype)).to(dtype)
    x = few.double().numpy()
    t = few.repeat(-(-n // len(few)), 1)[:n].cuda()
    y = rng.integers(0, v, len(few))
    y[::4] = v // 2
    for scale in (1.0, 0.7, 2.5):
        print("far logits", n, v, kind, scale, flush=True)
        got = run(lib, t, np.resize(y, n), 5, scale)
        ref = reference(x, y, 5, scale)
        many = np.resize(np.arange(len(few)), n)
        check_scores(got, {k: a[many] for k, a in ref.items()}, x[many], scale)


def test_the_smallest_and_largest_scales(lib):
    import torch
    x = np.array([[0.0, -1e-3, 2e-3, 2e-3], [5.0, 1.0, -3.0, 5.0], [1e30, -1e30, 1e30, 3e38]])
    t = torch.from_numpy(x).float().cuda()
    x = t.double().cpu().numpy()
    y = np.array([1, 0, 3])
    for scale in (LARGEST, 1e30, 1e-30, 1e-38):
        s = float(np.float32(scale))
        check_scores(run(lib, t, y, 2, s), reference(x, y, 2, s), x, s)


def check_gradient(got, x, y, ids, g, scale, lse, dtype):
    import torch
    n, v = x.shape
    top = x.max(1, keepdims=True)
    ref = lmo.scores_bwd(x - top, y, ids, scale=scale, **g)
    ref[lse == -np.inf] = 0
    log_l = lmo.scores(x - top, scale=scale)["lse"][:, None]
    logp = (x - top) * scale - log_l
    p, D = np.exp(logp), spread(x, scale)[:, None]
    far = (np.abs(lse) > 4096)[:, None]
    p_error = 4 * U * D + (v + 16) * U + np.where(far, 0, 4 * U * (np.where(far, 0, np.abs(lse)[:, None]) + D + np.where(p > 0, np.abs(np.where(p > 0, logp, 0)), 0)))
    named = np.zeros((n, v))
    for i in range(n):
        if 0 <= y[i] < v:
            named[i, y[i]] += abs(g["g_logp"][i])
        for j, a in zip(ids[i], g["g_top"][i]):
            named[i, j] += abs(a)
    size = np.abs(g["g_logp"])[:, None] + np.abs(g["g_lse"])[:, None] + np.abs(g["g_top"]).sum(1, keepdims=True)
    logs = np.where(p > 0, np.abs(np.where(p > 0, logp, 0)), 0) + math.log(v) + 1
    by_entropy = np.abs(g["g_entropy"])[:, None] * logs
    # p, log p + entropy and the sums each with their errors
    tol = scale * 2.0 ** -126 * (size + by_entropy) + scale * (p * (size + by_entropy) * (p_error + 16 * U) + p * np.abs(g["g_entropy"])[:, None] * (p_error + (2 * (v + 8) * U + 8 * U * D) * logs) + 12 * U * (named + p * size))
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol) + 2.0 ** -134
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol + 2.0 ** -140).all(), (np.argwhere(np.abs(got - ref) > tol + 2.0 ** -140)[:5].tolist(), float((np.abs(got - ref) - tol).max()))


@pytest.mark.parametrize("kinds", ["bf16 bf16", "f32 f32", "bf16 f32"])
@pytest.mark.parametrize("v", [300, 5003, 20011])                                # a wave a row; work-groups of one and of three parts
def test_gradient(lib, v, kinds):
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 96100 + v))
    types = [torch.bfloat16 if k == "bf16" else torch.float32 for k in kinds.split()]
    x16 = torch.from_numpy(rows_of(rng, v, types[0])).to(types[0])
    x, t, n = x16.double().numpy(), x16.cuda(), len(x16)
    y = rng.integers(0, v, n)
    for scale in (1.0, 2.5):
        s = run(lib, t, y, 5, scale)
        f32 = lambda *shape: rng.standard_normal(shape).astype(np.float32)
        g = {"g_logp": f32(n), "g_lse": f32(n), "g_entropy": f32(n), "g_top": f32(n, 5)}
        cuda = lambda a: torch.from_numpy(a).cuda()
        shp = lib.scores_shape(n, v, 5, scale)
        args = dict(y=cuda(y), entropy=cuda(s["entropy"]), top_ids=cuda(s["top_ids"]), **{k: cuda(a) for k, a in g.items()})
        out = torch.full((n, v), 7.0, device="cuda", dtype=types[1])
        print("far gradient", v, kinds, scale, flush=True)
        lib.burst_lm_head_scores_bwd(shp, t, cuda(s["lse"]), out, **args)
        torch.cuda.synchronize()
        check_gradient(out.double().cpu().numpy(), x, y, s["top_ids"], g, scale, s["lse"], types[1])
        if types[0] == types[1]:
            own = t.clone()
            lib.burst_lm_head_scores_bwd(shp, own, cuda(s["lse"]), own, **args)     # in the logits' place
            assert torch.equal(own, out)


def test_rows_beside_far_ones_keep_their_bits(lib):
    """Rows of ordinary logits among far ones, and rows of anything that a Lse of -inf leaves out."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 96200))
    n = 12
    for v in (300, 20011):
        t = torch.from_numpy(rng.standard_normal((n, v)) * 3).to(torch.bfloat16).cuda()
        y, shp, ones = torch.from_numpy(rng.integers(0, v, n)).cuda(), lib.scores_shape(n, v), torch.ones(n, device="cuda")

        def grad(x, lse):
            d = torch.empty_like(x)
            lib.burst_lm_head_scores_bwd(shp, x, lse, d, y=y, entropy=ones, g_logp=ones, g_entropy=ones)
            return d
        lse = torch.empty(n, device="cuda")
        lib.burst_lm_head_scores(shp, t, lse=lse, workspace=torch.empty(lib.burst_lm_head_scores_workspace_bytes(shp), device="cuda", dtype=torch.uint8))
        want = grad(t, lse)
        far, far_lse = t.clone(), lse.clone()
        far[1::3], far_lse[1::3] = -1e30, -1e30
        far[2], far[5], far[8, ::2], far_lse[2::3] = math.inf, math.nan, lowest(torch.bfloat16), -math.inf
        got = grad(far, far_lse)
        assert torch.equal(got[0::3], want[0::3]) and (got[2::3] == 0).all() and torch.isfinite(got).all()
