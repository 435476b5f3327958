"""Scores of tokens from logits, and the gradient of the logits, on the GPU against the fp64 reference.

Tolerances, with u = 2^-24, x = scale * logits and M the largest |x| of a row: its exponent to base 2 is off by 3 u M (two roundings and that of the maximum), the sum of v
exponentials by (v + 8) u of itself; so Lse by e = 3 u M + (v + 8) u + 2 u |Lse|.  A log probability is a difference of two numbers off by e and u M: 2 u M + e.  The
entropy is a sum of p |log p| over p with the same relative errors, and log l - w / l in base 2: (2 (v + 8) u + 6 u M) (1 + E), E the sum of p |x - max| (at most log v + entropy).
A gradient is scale times a sum of products of numbers off so, relative to the sum of their sizes, and half a step of its type."""
import math

import numpy as np
import pytest

from oracle import lm_head_oracle as lmo
from paper_2509_19836_amd import workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(rng, n, v, dtype, allowed=1.0, pad=0, spread=2.0):
    """Logits in rows of v + pad elements (padding NaN) on the GPU, and their values."""
    import torch
    x = rng.standard_normal((n, v)).astype(np.float32)
    x = spread * x + 0.5 * np.abs(x) * x
    if allowed < 1:
        x[rng.random((n, v)) >= allowed] = -np.inf
        x[:, v // 2] = 0.25
    wide = torch.full((n, v + pad), float("nan"), device="cuda", dtype=dtype)
    t = wide[:, :v]
    t.copy_(torch.from_numpy(x))
    return t, t.double().cpu().numpy()


def targets(rng, n, v):
    y = rng.integers(0, v, n)
    y[rng.random(n) < 0.2] = rng.choice([-1, v, -100, 2 ** 40])
    return y


def run(lib, t, y, n_top, scale, want=("logp", "lse", "entropy", "top_logp", "top_ids")):
    import torch
    n, v = t.shape
    shp = lib.scores_shape(n, v, n_top, scale)
    kinds = {"logp": ((n,), torch.float32), "lse": ((n,), torch.float32), "entropy": ((n,), torch.float32), "top_logp": ((n, n_top), torch.float32),
             "top_ids": ((n, n_top), torch.int64)}
    out = {k: torch.full(s, 77, device="cuda", dtype=d) for k, (s, d) in kinds.items() if k in want and (n_top > 0 or not k.startswith("top"))}
    ws = torch.full((lib.burst_lm_head_scores_workspace_bytes(shp),), 255, device="cuda", dtype=torch.uint8)
    lib.burst_lm_head_scores(shp, t, y=torch.from_numpy(y).cuda() if "logp" in out else None, workspace=ws, **out)
    torch.cuda.synchronize()
    return {k: x.cpu().numpy() for k, x in out.items()}


def check(got, ref, x, scale):
    v = x.shape[1]
    M = scale * np.abs(np.where(np.isinf(x), 0, x)).max(1)
    e = 3 * U * M + (v + 8) * U + 2 * U * np.abs(np.where(np.isinf(ref["lse"]), 0, ref["lse"]))

    def near(a, b, tol):
        same = (a == b) | (np.abs(np.where(np.isinf(a), 0, a) - np.where(np.isinf(b), 0, b)) <= tol) & np.isfinite(a) & np.isfinite(b)
        assert same.all(), (a[~same][:5], b[~same][:5])
    near(got["lse"], ref["lse"], e)
    if "logp" in got:
        near(got["logp"], ref["logp"], 2 * U * M + e + 2 * U * np.abs(np.where(np.isinf(ref["logp"]), 0, ref["logp"])))
    if "entropy" in got:
        near(got["entropy"], ref["entropy"], (2 * (v + 8) * U + 6 * U * M) * (1 + math.log(v) + ref["entropy"]))
    if "top_ids" in got:
        assert np.array_equal(got["top_ids"], ref["top_ids"])
        near(got["top_logp"], ref["top_logp"], (2 * U * M + e)[:, None] + 2 * U * np.abs(np.where(np.isinf(ref["top_logp"]), 0, ref["top_logp"])))


SIZES = [(1, 1, 1), (1, 2, 2), (3, 7, 5), (5, 64, 64), (2, 200, 64), (4, 257, 1), (7, 1000, 20), (1, 5003, 8), (3, 40000, 33), (600, 300, 4), (2100, 130, 3), (515, 2051, 9)]


@pytest.mark.parametrize("n,v,n_top", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_scores_against_the_reference(lib, n, v, n_top, kind):
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 93000 + n + v))
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    for scale, allowed, pad in ((1.0, 1.0, 0), (0.7, 0.3, 3), (2.5, 0.02, 8)):
        t, x = make(rng, n, v, dtype, allowed, pad)
        y = targets(rng, n, v)
        print("scores", n, v, n_top, kind, scale, allowed, pad, flush=True)
        ref = lmo.scores(x, y, n_top, scale)
        got = run(lib, t, y, n_top, scale)
        check(got, ref, x, scale)
        part = run(lib, t, y, 0, scale)
        assert all(np.array_equal(part[k], got[k], equal_nan=True) for k in part)             # without the likeliest words the same bits


@pytest.mark.parametrize("n,v", [(3, 110000), (3, 70000), (520, 3000), (2050, 400), (40, 9000)])
def test_every_way_of_dealing_a_row(lib, n, v):
    """A wave, four, sixteen, several work-groups: by burst_lm_head_scores_plan, the same words everywhere."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 93100 + n))
    plan = lib.burst_lm_head_scores_plan(lib.scores_shape(n, v, 10))
    print("plan", n, v, plan, flush=True)
    t, x = make(rng, n, v, torch.bfloat16)
    y = targets(rng, n, v)
    got = run(lib, t, y, 10, 1.0)
    check(got, lmo.scores(x, y, 10, 1.0), x, 1.0)
    again = run(lib, t, y, 10, 1.0)
    assert all(np.array_equal(again[k], got[k]) for k in got)


def test_plans_cover_every_kernel(lib):
    plans = {lib.burst_lm_head_scores_plan(lib.scores_shape(n, v, 10)) for n, v in ((3, 110000), (3, 70000), (520, 3000), (2050, 400), (40, 9000))}
    assert {w for w, _ in plans} == {1, 4, 16} and {s > 1 for _, s in plans} == {False, True}


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 700, 2100])
def test_order_of_hard_rows(lib, kind, n):
    """Rows that rise, fall, are all alike, hold two values, both zeros, infinities below, one word, or their largest numbers side by side or a lane apart."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 93200 + n))
    v, dtype = 3001, torch.bfloat16 if kind == "bf16" else torch.float32
    rows = [np.linspace(-3, 30, v), np.linspace(30, -3, v), np.full(v, 1.5), rng.integers(0, 2, v) * 1.0, np.where(rng.random(v) < 0.5, 0.0, -0.0),
            np.full(v, -np.inf), np.where(np.arange(v) == 1234, 3.0, -np.inf), np.where(np.arange(v) < 2, -2.0, -np.inf), np.arange(v) % 64 * 0.1,
            np.arange(v) // 64 * 0.25, np.where(np.arange(v) >= v - 70, 9.0, rng.standard_normal(v)), np.where(np.arange(v) % 512 < 8, 9.0, rng.standard_normal(v)),
            -1e30 * rng.random(v), rng.standard_normal(v) * 1e-30]
    x = np.stack([rows[i % len(rows)] for i in range(n * (7 if n == 2 else 1))])
    t = torch.from_numpy(x).cuda().to(dtype)
    x = t.double().cpu().numpy()
    few = x[:len(rows)]
    ref = lmo.scores(few, np.zeros(len(few), np.int64), 64, 1.0)
    got = run(lib, t, np.zeros(len(x), np.int64), 64, 1.0)
    assert np.array_equal(got["top_ids"][:len(few)], ref["top_ids"])
    repeat = got["top_ids"].reshape(len(x), 64)
    for i in range(len(rows), len(x)):
        assert np.array_equal(repeat[i], ref["top_ids"][i % len(rows)])
    keep = [i for i in range(len(few)) if i != 12]                            # (1e30: logits whose fp32 exponents say nothing of the sums)
    check({k: a[:len(few)][keep] for k, a in got.items()}, {k: a[keep] for k, a in ref.items()}, few[keep], 1.0)


@pytest.mark.parametrize("n,v", [(2, 32768), (600, 16384), (2100, 20500)])
def test_large_numbers_in_few_places(lib, n, v):
    """All large numbers where few threads of the kernels read: every stretch of 512 words, or of 256, begins with some; or the first 2048 words."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 93250 + n))
    j = np.arange(v)
    for dtype in (torch.bfloat16, torch.float32):
        for where in (j % 512 < 8, j % 256 < 4, (j < 2048) & (j % 512 < 504), (j < 2048) & (j % 256 < 252), j % 2048 < 480):
            base = np.where(where, 20.0 + rng.random(v), rng.standard_normal(v))
            t = torch.from_numpy(base).cuda().to(dtype)
            x = t.double().cpu().numpy()
            want = np.lexsort((j, -x))[:64]
            got = run(lib, t[None].expand(n, -1).contiguous(), np.zeros(n, np.int64), 64, 1.0)
            assert (got["top_ids"] == want).all()


@pytest.mark.parametrize("n,v", [(3, 5000), (2100, 100)])
def test_not_finite(lib, n, v):
    """A NaN or +inf among a token's logits: NaN for its scores, words for its ids; the others as without it."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 93300))
    t, x = make(rng, n, v, torch.float32)
    y = rng.integers(0, v, n)
    clean = run(lib, t, y, 6, 1.0)
    t[1, v // 3], t[2, v // 2] = float("nan"), float("inf")
    got = run(lib, t, y, 6, 1.0)
    for k, a in got.items():
        assert np.array_equal(a[0], clean[k][0]) and np.array_equal(a[3:], clean[k][3:])
        if k != "top_ids":
            assert np.isnan(a[1]).all() and not np.isfinite(a[2]).any()
    assert ((got["top_ids"] >= 0) & (got["top_ids"] < v)).all() and got["top_ids"][2, 0] == v // 2
    t[1] = float("nan")
    ids = run(lib, t, y, 6, 1.0)["top_ids"][1]
    assert ((ids >= 0) & (ids < v)).all()


def test_outputs_one_by_one_and_no_tokens(lib):
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 93400))
    t, x = make(rng, 9, 777, torch.bfloat16)
    y = targets(rng, 9, 777)
    whole = run(lib, t, y, 5, 1.3)
    for k in whole:
        assert np.array_equal(run(lib, t, y, 5, 1.3, (k,))[k], whole[k])
    lib.burst_lm_head_scores(lib.scores_shape(0, 777, 5), t[:0], lse=torch.empty(0, device="cuda"))
    lib.burst_lm_head_scores_bwd(lib.scores_shape(0, 777, 5), t[:0], torch.empty(0, device="cuda"), t[:0], g_lse=torch.empty(0, device="cuda"))


GRADS = [(1, 1, 1), (2, 9, 3), (3, 64, 7), (5, 1001, 64), (2, 30011, 20), (300, 257, 5)]


@pytest.mark.parametrize("n,v,n_top", GRADS)
@pytest.mark.parametrize("kinds", ["bf16 bf16", "bf16 f32", "f32 f32", "f32 bf16"])
def test_gradient_against_the_reference(lib, n, v, n_top, kinds):
    """All gradients that come in, each alone, words named twice and words that are none, strided rows of both whose rest stays as it is."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 94000 + n + v))
    types = [torch.bfloat16 if k == "bf16" else torch.float32 for k in kinds.split()]
    for scale, allowed, pads in ((1.0, 1.0, (0, 0)), (0.7, 0.4, (3, 3)), (1.6, 1.0, (8, 5))):
        t, x = make(rng, n, v, types[0], allowed, pads[0])
        y = targets(rng, n, v)
        s = run(lib, t, y, n_top, scale)
        ids = s["top_ids"].copy()
        if n_top > 2:
            ids[0, 1], ids[0, 2], ids[-1, 0] = ids[0, 0], -1, v + 5
            ids[-1, 1] = y[-1] if 0 <= y[-1] < v else ids[-1, 2]
        f32 = lambda *shape: rng.standard_normal(shape).astype(np.float32)
        g = {"g_logp": f32(n), "g_lse": f32(n), "g_entropy": f32(n), "g_top": f32(n, n_top)}
        cuda = lambda a: torch.from_numpy(a).cuda()
        print("gradient", n, v, n_top, kinds, scale, flush=True)
        for use in (list(g),) + tuple([k] for k in g):
            wide = torch.full((n, v + pads[1]), 7.0, device="cuda", dtype=types[1])
            part = {k: g[k] for k in use}
            lib.burst_lm_head_scores_bwd(lib.scores_shape(n, v, n_top, scale), t, cuda(s["lse"]), wide[:, :v], y=cuda(y) if "g_logp" in use else None,
                                         entropy=cuda(s["entropy"]) if "g_entropy" in use else None, top_ids=cuda(ids) if "g_top" in use else None,
                                         **{k: cuda(a) for k, a in part.items()})
            torch.cuda.synchronize()
            ref = lmo.scores_bwd(x, y, ids, scale=scale, **part)
            # each p is off by (3 u M + (v + 8) u) of itself, log p + entropy by as much and a rounding; sums of up to n_top + 3 numbers
            M = scale * np.abs(np.where(np.isinf(x), 0, x)).max(1, keepdims=True)
            p = np.exp(x * scale - lmo.scores(x, scale=scale)["lse"][:, None])
            named = np.zeros((n, v))
            for i in range(n):
                if "g_logp" in use and 0 <= y[i] < v:
                    named[i, y[i]] += abs(g["g_logp"][i])
                for j, a in zip(ids[i], g["g_top"][i]) if "g_top" in use else ():
                    if 0 <= j < v:
                        named[i, j] += abs(a)
            size = sum(np.abs(part[k]).reshape(n, -1).sum(1, keepdims=True) for k in use if k != "g_entropy") if use != ["g_entropy"] else np.zeros((n, 1))
            logs = np.where(p > 0, np.abs(np.where(np.isinf(x), 0, x) * scale) + M, 0) + math.log(v) + 1
            if "g_entropy" in use:
                size = size + np.abs(g["g_entropy"])[:, None] * logs
            tol = scale * ((8 * U * M + (2 * v + 40) * U) * p * (size + np.abs(g["g_entropy"])[:, None] * 8 * ("g_entropy" in use)) + (n_top + 8) * U * (named + p * size))
            if types[1] == torch.bfloat16:
                tol = tol + 2.0 ** -8 * (np.abs(ref) + tol) + 2.0 ** -134
            got = wide[:, :v].double().cpu().numpy()
            assert (np.abs(got - ref) <= tol + 2.0 ** -140).all(), (use, float((np.abs(got - ref) - tol).max()))
            assert (wide[:, v:] == 7).all()


def test_gradient_in_place_and_where_all_is_masked(lib):
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 94100))
    for n, v, dtype in ((5, 20011, torch.bfloat16), (4, 9000, torch.float32)):
        t, x = make(rng, n, v, dtype)
        t[1] = -math.inf
        y = rng.integers(0, v, n)
        s = run(lib, t, y, 7, 1.1)
        cuda = lambda a: torch.from_numpy(a).cuda()
        args = dict(y=cuda(y), entropy=cuda(s["entropy"]), top_ids=cuda(s["top_ids"]))
        args.update({k: torch.randn(n, device="cuda") for k in ("g_logp", "g_lse", "g_entropy")}, g_top=torch.randn(n, 7, device="cuda"))
        out, shp = torch.empty_like(t), lib.scores_shape(n, v, 7, 1.1)
        lib.burst_lm_head_scores_bwd(shp, t, cuda(s["lse"]), out, **args)
        lib.burst_lm_head_scores_bwd(shp, t, cuda(s["lse"]), t, **args)
        assert torch.equal(out, t) and (out[1] == 0).all() and torch.isfinite(out).all()


def test_gradient_by_differences(lib):
    """Differences of the scores themselves, on the GPU, along random directions."""
    import torch
    torch.manual_seed(5)
    n, v, h = 4, 300, 2.0 ** -6
    x = torch.randn(n, v, device="cuda") * 2
    y = torch.randint(0, v, (n,), device="cuda")
    shp = lib.scores_shape(n, v, 3, 0.8)
    f = lambda *s: torch.empty(*s, device="cuda")

    def scores(z):
        out = dict(logp=f(n), lse=f(n), entropy=f(n))
        ws = torch.empty(lib.burst_lm_head_scores_workspace_bytes(shp), device="cuda", dtype=torch.uint8)
        lib.burst_lm_head_scores(shp, z, y=y, workspace=ws, **out)
        return out
    g = {k: torch.randn(n, device="cuda") for k in ("logp", "lse", "entropy")}
    s, d = scores(x), f(n, v)
    lib.burst_lm_head_scores_bwd(shp, x, s["lse"], d, y=y, entropy=s["entropy"], g_logp=g["logp"], g_lse=g["lse"], g_entropy=g["entropy"])
    for _ in range(4):
        e = torch.randn(n, v, device="cuda")
        up, down = scores(x + h * e), scores(x - h * e)
        want = sum((g[k].double() * (up[k].double() - down[k].double())).sum(0) for k in g) / (2 * h)
        # third derivatives of size 1 to 4 times h^2 / 6 a token, roundings 2^-21 / h
        assert abs((d.double() * e.double()).sum() - want) <= 4 * n * 4 * h * h / 6 * float(e.abs().max()) ** 3 + 3 * n * 2.0 ** -21 / h


def test_graph_and_streams(lib):
    """Scores and their gradient captured, replayed with other logits between eager calls; two calls on streams of their own."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 94200))
    n, v = 6, 110001
    t, _ = make(rng, n, v, torch.bfloat16)
    y = torch.from_numpy(rng.integers(0, v, n)).cuda()
    shp = lib.scores_shape(n, v, 12)
    assert lib.burst_lm_head_scores_plan(shp)[1] > 1
    ws = torch.empty(lib.burst_lm_head_scores_workspace_bytes(shp), device="cuda", dtype=torch.uint8)
    f = lambda: dict(logp=torch.empty(n, device="cuda"), lse=torch.empty(n, device="cuda"), entropy=torch.empty(n, device="cuda"),
                     top_logp=torch.empty(n, 12, device="cuda"), top_ids=torch.empty(n, 12, device="cuda", dtype=torch.int64))
    out, d, g = f(), torch.empty_like(t), torch.randn(n, device="cuda")

    def calls(o, grad, w, stream=None):
        lib.burst_lm_head_scores(shp, t, y=y, workspace=w, stream=stream, **o)
        lib.burst_lm_head_scores_bwd(shp, t, o["lse"], grad, y=y, entropy=o["entropy"], g_logp=g, g_entropy=g, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(out, d, ws)
    for turn in range(4):
        t.copy_(torch.randn(n, v, device="cuda") * (turn + 1))
        graph.replay()
        got, got_d = {k: x.clone() for k, x in out.items()}, d.clone()
        eager, eager_d = f(), torch.empty_like(t)
        calls(eager, eager_d, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], eager[k]) for k in got) and torch.equal(got_d, eager_d)
    streams = [torch.cuda.Stream() for _ in range(2)]
    parts = [(f(), torch.empty_like(t), torch.empty_like(ws)) for _ in streams]
    torch.cuda.synchronize()
    for s, p in zip(streams, parts):
        calls(*p, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for o, grad, _ in parts:
        assert all(torch.equal(o[k], eager[k]) for k in o) and torch.equal(grad, eager_d)


def test_rows_beyond_32_bits(lib):
    """Rows 2 GiB elements from each other."""
    import torch
    big = torch.empty((1 << 32) + (1 << 20), device="cuda", dtype=torch.bfloat16)
    t = big.as_strided((3, 5000), (1 << 31, 1))
    x = torch.randn(3, 5000, device="cuda").to(torch.bfloat16)
    t.copy_(x)
    y = np.array([3, 4999, 17])
    a, b = run(lib, t, y, 4, 1.0), run(lib, x, y, 4, 1.0)
    assert all(np.array_equal(a[k], b[k]) for k in a)
    cuda = lambda z: torch.from_numpy(z).cuda()
    out, shp = torch.empty_like(x), lib.scores_shape(3, 5000, 4)
    lib.burst_lm_head_scores_bwd(shp, x, cuda(a["lse"]), out, y=cuda(y), g_logp=torch.ones(3, device="cuda"))
    lib.burst_lm_head_scores_bwd(shp, t, cuda(a["lse"]), t, y=cuda(y), g_logp=torch.ones(3, device="cuda"))
    assert torch.equal(out, t)
