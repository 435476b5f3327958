"""Every kernel that burst_attn_decode may take, at its edges: head widths, types, groups of up to and over 16 query heads, pages of a multiple of 16
rows and of any, work dealt to shares and not, key heads one by one and side by side.  Pages are shared between sequences, as those
of a common prompt are, so that the caches stay small while the rows are many; sampled sequences are held against the fp64 reference
with the tolerances of tests/test_gpu_paged_cache.py."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import test_gpu_paged_cache as tp

pytestmark = pytest.mark.gpu

# (mode, batch, kv_heads, longest sequence): few short rows; rows beyond 512 KiB a head; 4 units and more for every work-group that fits
MODES = {"direct": (9, 4, 300), "dealt": (5, 3, 4500), "beside": (70, 4, 4600)}


def _pool(lib, rng, rows, page_rows, Hkv, d, f8, pool_rows=3000):
    """Sequences whose pages all come from one pool."""
    P = tp.Paged(lib, rng, [pool_rows], page_rows, Hkv, d, f8)
    cols = -(-max(rows) // page_rows)
    P.table = rng.integers(0, P.n_pages, (len(rows), cols)).astype(np.int32)
    P.rows = list(rows)
    import torch
    put = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    P.put_table, P.put_rows = put(P.table), put(np.array(rows, np.int32))
    P.cache = lib.paged_cache(P.dev["k"], P.dev["v"], P.put_table, P.put_rows, put(P.k_scale), put(P.v_scale))
    return P


@pytest.mark.parametrize("page_rows", [16, 12])
@pytest.mark.parametrize("group", [3, 21])
@pytest.mark.parametrize("d,f8", [(128, False), (128, True), (64, False), (64, True)])
@pytest.mark.parametrize("mode", list(MODES))
def test_kernel(lib, mode, d, f8, group, page_rows):
    import torch
    B, Hkv, longest = MODES[mode]
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 87000 + d + group + page_rows + f8))
    rows = rng.integers(0, longest, B).tolist()
    rows[0], rows[1], rows[-1] = longest, 0, longest - 33
    first = [0 if b % 3 else max(0, r - 77) for b, r in enumerate(rows)]
    P = _pool(lib, rng, rows, page_rows, Hkv, d, f8)
    q, q_host = tp.queries(rng, B, Hkv * group, d)
    shp = lib.shape(B, Hkv * group, Hkv, d, 1, longest, d ** -0.5)
    shares, heads, direct = lib.burst_attn_decode_plan(shp, P.cache)
    assert direct == (mode == "direct") and (heads > 1) == (mode == "beside")
    print(f"decode {mode} d={d} f8={f8} group={group} pages of {page_rows}: {shares} shares, {heads} heads", flush=True)
    o, lse = tp.run_decode(lib, P, q, d ** -0.5, longest, first)
    some = [0, 1, 2, 3, B - 2, B - 1]
    ref = co.decode(q_host[some], P.host["k"], P.host["v"], P.table[some], [rows[b] for b in some], d ** -0.5, [first[b] for b in some], None,
                    P.k_scale, P.v_scale)
    tp.check_decode(o[some], lse[some], ref, longest, d)
    o2, lse2 = tp.run_decode(lib, P, q, d ** -0.5, longest, first)        # the same bits again
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("B", [63, 64, 65, 256, 257, 513])
def test_scan_over_the_sequences(lib, B):
    """Batches around the sizes at which the scan changes: the sequences' lengths are all that decides who finds what."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 88000 + B))
    rows = rng.integers(0, 400, B).tolist()
    rows[B // 2] = 9000                                                    # (dealt: more than 512 KiB a head)
    P = _pool(lib, rng, rows, 16, 1, 64, False)
    q, q_host = tp.queries(rng, B, 2, 64)
    assert not lib.burst_attn_decode_plan(lib.shape(B, 2, 1, 64, 1, 9000, 0.125), P.cache)[2]
    o, lse = tp.run_decode(lib, P, q, 0.125, 9000)
    tp.check_decode(o, lse, co.decode(q_host, P.host["k"], P.host["v"], P.table, rows, 0.125), 9000, 64)


@pytest.mark.parametrize("mode", ["direct", "dealt"])
def test_strided_views_and_one_table_for_all(lib, mode):
    """q, o and lse as parts of larger tensors, whose rest stays as it is; one row of the table for all sequences (stride 0)."""
    import torch
    B, Hkv, longest = MODES[mode]
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 88100))
    rows = rng.integers(1, longest, B).tolist()
    rows[0] = longest
    d, Hq = 128, Hkv * 2
    P = _pool(lib, rng, rows, 16, Hkv, d, False)
    P.table = np.repeat(P.table[:1], B, 0)
    one = torch.from_numpy(P.table[:1].copy()).cuda().expand(B, -1)
    cache = lib.paged_cache(P.dev["k"], P.dev["v"], one, P.put_rows)
    q, q_host = tp.queries(rng, B, Hq, d)
    wide_q = torch.full((B, 3, Hq + 5, d), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide_q[:, 1:2, 2:2 + Hq] = q
    wide_o, wide_lse = torch.full((B, 2, Hq + 3, d), 7.0, device="cuda"), torch.full((B, Hq + 1, 6), 7.0, device="cuda")
    shp = lib.shape(B, Hq, Hkv, d, 1, longest, 0.09)
    ws = torch.empty(lib.burst_attn_decode_workspace_bytes(shp) + 256, device="cuda", dtype=torch.uint8)
    lib.burst_attn_decode(shp, cache, wide_q[:, 1:2, 2:2 + Hq], wide_o[:, :1, 1:1 + Hq], wide_lse[:, :Hq, 3:4], ws)
    torch.cuda.synchronize()
    tp.check_decode(wide_o[:, :1, 1:1 + Hq], wide_lse[:, :Hq, 3:4], co.decode(q_host, P.host["k"], P.host["v"], P.table, rows, 0.09), longest, d)
    assert (wide_o[:, 1:] == 7).all() and (wide_o[:, :, 0] == 7).all() and (wide_o[:, :, Hq + 1:] == 7).all()
    assert (wide_lse[:, Hq:] == 7).all() and (wide_lse[:, :, :3] == 7).all() and (wide_lse[:, :, 4:] == 7).all()


def test_two_graphs_one_workspace(lib):
    """Two captured calls that share a workspace, replayed in turn on one stream with eager calls and changing lengths between: the eager
    results, every time."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 88200))
    B, Hkv, longest = MODES["dealt"]
    P = _pool(lib, rng, [longest] * B, 16, Hkv, 64, False)
    shp = lib.shape(B, Hkv * 4, Hkv, 64, 1, longest, 0.125)
    ws = torch.full((lib.burst_attn_decode_workspace_bytes(shp),), 255, device="cuda", dtype=torch.uint8)
    q = [tp.queries(rng, B, Hkv * 4, 64)[0] for _ in range(2)]
    o = [torch.zeros(B, 1, Hkv * 4, 64, device="cuda") for _ in range(2)]
    lse = [torch.zeros(B, Hkv * 4, 1, device="cuda") for _ in range(2)]
    first = torch.zeros(B, dtype=torch.int32, device="cuda")
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            lib.burst_attn_decode(shp, P.cache, q[i], o[i], lse[i], ws, first_row=first)
    for turn in range(4):
        P.put_rows.copy_(torch.tensor(rng.integers(0, longest, B), dtype=torch.int32))
        first.copy_((P.put_rows * 0.3).to(torch.int32) * (turn % 2))
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        got = [(a.clone(), b.clone()) for a, b in zip(o, lse)]
        for i in range(2):
            lib.burst_attn_decode(shp, P.cache, q[i], o[i], lse[i], ws, first_row=first)
            torch.cuda.synchronize()
            assert torch.equal(o[i], got[i][0]) and torch.equal(lse[i], got[i][1])


def test_streams_of_their_own(lib):
    """Calls on two streams at once, each with its workspace, against the calls one after the other."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 88300))
    B, Hkv, longest = MODES["dealt"]
    P = _pool(lib, rng, [longest - 7 * b for b in range(B)], 16, Hkv, 128, True)
    q = [tp.queries(rng, B, Hkv * 2, 128)[0] for _ in range(2)]
    alone = [tp.run_decode(lib, P, x, 0.09, longest) for x in q]
    shp = lib.shape(B, Hkv * 2, Hkv, 128, 1, longest, 0.09)
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = []
    torch.cuda.synchronize()
    for s, x in zip(streams, q):
        with torch.cuda.stream(s):
            ws = torch.empty(lib.burst_attn_decode_workspace_bytes(shp), device="cuda", dtype=torch.uint8)
            o, lse = torch.empty(B, 1, Hkv * 2, 128, device="cuda"), torch.empty(B, Hkv * 2, 1, device="cuda")
            for _ in range(5):
                lib.burst_attn_decode(shp, P.cache, x, o, lse, ws, stream=s.cuda_stream)
            out.append((o, lse, ws))
    torch.cuda.synchronize()
    for (o, lse, _), (o1, lse1) in zip(out, alone):
        assert torch.equal(o, o1) and torch.equal(lse, lse1)


@pytest.mark.parametrize("in_type,out_type", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_large_rotations_are_the_small_ones(lib, in_type, out_type):
    """More than the chip keeps (other instructions move it): the same bits as the rows in pieces."""
    import torch
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    n, Hq, Hkv, d = 24000, 20, 4, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k = (torch.randn(1, n, h, d, generator=gen, device="cuda").to(types[in_type]) for h in (Hq, Hkv))
    pos = torch.randint(0, 1 << 20, (1, 1, n), generator=gen, device="cuda", dtype=torch.int32)
    freq = torch.rand(64, generator=gen, device="cuda")
    out = [torch.empty_like(t, dtype=types[out_type]) for t in (q, k)]
    assert sum(t.numel() * t.element_size() for t in (q, k, *out)) > 1 << 28
    lib.burst_attn_rope(lib.shape(1, Hq, Hkv, d, n, 0, 1.0), lib.rope(pos, freq), q, out[0], k, out[1])
    for i in range(0, n, 6000):
        part = slice(i, i + 6000)
        qo, ko = (torch.empty_like(t[:, part]) for t in out)
        lib.burst_attn_rope(lib.shape(1, Hq, Hkv, d, 6000, 0, 1.0), lib.rope(pos[:, :, part], freq), q[:, part], qo, k[:, part], ko)
        assert torch.equal(qo, out[0][:, part]) and torch.equal(ko, out[1][:, part])


@pytest.mark.parametrize("f8", [False, True])
def test_large_appends_are_the_small_ones(lib, f8):
    import torch
    n, Hq, Hkv, d = 16000, 40, 8, 128
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(1, n, h, d, generator=gen, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, 1 << 20, (1, 1, n), generator=gen, device="cuda", dtype=torch.int32)
    freq, table = torch.rand(64, generator=gen, device="cuda"), torch.randperm(1000, generator=gen, device="cuda").to(torch.int32)[None]
    results = []
    for step in (n, 2000):
        pages = [torch.zeros(1000, 16, Hkv, d, device="cuda", dtype=torch.float8_e4m3fn if f8 else torch.bfloat16) for _ in range(2)]
        rows, q_out = torch.zeros(1, device="cuda", dtype=torch.int32), torch.zeros_like(q)
        cache = lib.paged_cache(*pages, table, rows)
        for i in range(0, n, step):
            part = slice(i, i + step)
            rows += step
            lib.burst_attn_cache_append(lib.shape(1, Hq, Hkv, d, step, 0, 1.0), cache, k[:, part], v[:, part], None,
                                        lib.rope(pos[:, :, part], freq), q[:, part], q_out[:, part])
        results.append([p.view(torch.uint8) for p in pages] + [q_out])
    for a, b in zip(*results):
        assert torch.equal(a, b)
