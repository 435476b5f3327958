"""Pages copied and rows moved to the front, in all layers of a model at once: every byte of the caches as the reference has it."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl

pytestmark = pytest.mark.gpu

LAYOUTS = [(5, 16, 2, 64, False, False), (3, 64, 8, 128, False, True), (4, 7, 3, 128, True, False), (9, 1, 5, 64, True, True), (2, 256, 1, 128, False, False),
           (40, 12, 4, 64, False, True)]


def numbers(rng, n_layers, n_pages, page_rows, Hkv, d, f8, by_head):
    """Layers of keys and values with random bytes (NaN among them), as tensors [pages, rows, heads, head_dim] and as whole numbers on the host."""
    import torch
    dev, host = [], []
    for _ in range(2 * n_layers):
        bits = rng.integers(0, 256 if f8 else 65536, (n_pages, Hkv, page_rows, d) if by_head else (n_pages, page_rows, Hkv, d)).astype(np.uint8 if f8 else np.uint16)
        t = torch.from_numpy(bits.view(np.uint8 if f8 else np.int16).copy()).cuda().view(torch.float8_e4m3fn if f8 else torch.bfloat16)
        dev.append(t.transpose(1, 2) if by_head else t)
        host.append(bits.transpose(0, 2, 1, 3) if by_head else bits)
    return dev, host


def read(t):
    import torch
    f8 = t.dtype == torch.float8_e4m3fn
    x = t.view(torch.uint8 if f8 else torch.int16).cpu().numpy()
    return x if f8 else x.view(np.uint16)


def handles(lib, dev, table, rows):
    import torch
    put = lambda a: torch.from_numpy(np.asarray(a, np.int32)).cuda()
    t, r = put(table), put(rows)
    return lib.cache_layers(lib.paged_cache(dev[2 * i], dev[2 * i + 1], t, r) for i in range(len(dev) // 2))


@pytest.mark.parametrize("n_layers,page_rows,Hkv,d,f8,by_head", LAYOUTS + [(70, 16, 2, 64, False, False)])
def test_copied_pages(lib, n_layers, page_rows, Hkv, d, f8, by_head):
    """Whole pages, parts, none; one source for several; counts out of range; pages that are none; a page to itself; more layers than a launch takes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 92000 + n_layers + d))
    n_pages = 24
    dev, host = numbers(rng, n_layers, n_pages, page_rows, Hkv, d, f8, by_head)
    moves = [(3, 10, page_rows), (3, 11, page_rows // 2), (4, 12, 1), (5, 13, 0), (6, 14, -3), (7, 15, page_rows + 100), (-1, 16, 5), (8, n_pages, 5), (8, -2, 5),
             (n_pages + 7, 17, 5), (9, 9, page_rows), (3, 18, page_rows - 1), (2 ** 31 - 1, 19, 3), (0, 23, page_rows)]
    layers = handles(lib, dev, [[0, 1]], [2])
    print("copy", n_layers, page_rows, Hkv, d, f8, by_head, flush=True)
    lib.burst_attn_cache_copy_pages(layers, torch.tensor(moves, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for t, h in zip(dev, host):
        assert np.array_equal(read(t), co.copy_pages(h, moves))
    lib.burst_attn_cache_copy_pages(layers, torch.zeros(0, 3, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("n_layers,page_rows,Hkv,d,f8,by_head", LAYOUTS + [(66, 16, 2, 64, False, False)])
@pytest.mark.parametrize("sq", [1, 6, 64])
def test_kept_rows(lib, n_layers, page_rows, Hkv, d, f8, by_head, sq):
    """Rows in any order, named twice, out of range; none kept, all; rows that lie in several pages or in none; counts out of range."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 92100 + n_layers + d + sq))
    B, longest = 7, 150
    cols = -(-longest // page_rows) + 1
    n_pages = B * cols + 1
    dev, host = numbers(rng, n_layers, n_pages, page_rows, Hkv, d, f8, by_head)
    table = rng.permutation(n_pages - 1)[:B * cols].reshape(B, cols).astype(np.int32)
    table[3, (100 - 1) // page_rows] = -1
    rows = [longest, sq, max(1, sq // 2), 100, 10 ** 6, 90, -3]
    new = [sq, sq, sq, min(sq, 3), 100, -5, sq]
    kept = [sq, (sq + 1) // 2, sq + 5, 3, max(1, sq - 1), 4, 2]
    source = rng.integers(-1, sq + 1, (B, sq))
    source[0] = rng.permutation(sq)                                            # every row is another's source and destination
    source[1] = np.sort(rng.integers(0, sq, sq))
    layers = handles(lib, dev, table, rows)
    put = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    print("keep", n_layers, page_rows, Hkv, d, f8, by_head, sq, flush=True)
    lib.burst_attn_cache_keep_rows(layers, put(source), put(kept), new_rows=put(new))
    torch.cuda.synchronize()
    want = [co.keep_rows(h, table, rows, source, new, kept) for h in host]
    for t, h in zip(dev, want):
        assert np.array_equal(read(t), h)
    want = [co.keep_rows(h, table, rows, np.repeat(source[:1], B, 0), [sq] * B, kept) for h in want]   # one list for all, all rows new
    lib.burst_attn_cache_keep_rows(layers, put(source[:1]).expand(B, -1), put(kept))
    torch.cuda.synchronize()
    for t, h in zip(dev, want):
        assert np.array_equal(read(t), h)


def test_strides_and_far_pages(lib):
    """Layers that lie in one tensor page by page, and pages beyond 32 bits from each other: nothing but the rows named changes."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 92200))
    L, n_pages, R, Hkv, d = 3, 6, 16, 2, 64
    flat = torch.from_numpy(rng.integers(0, 65536, (n_pages, L, 2, R + 1, Hkv, d + 8)).astype(np.uint16).view(np.int16)).cuda().view(torch.bfloat16)
    before = read(flat)
    dev = [flat[:, i, kv, :R, :, :d] for i in range(L) for kv in range(2)]
    table, rows = np.array([[4, 2, 0]], np.int32), [40]
    layers = handles(lib, dev, table, rows)
    put = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    lib.burst_attn_cache_copy_pages(layers, put([[4, 1, 9], [2, 3, 16]]))
    lib.burst_attn_cache_keep_rows(layers, put([[11, 3, 7, 0]]), put([3]), new_rows=put([4]))      # (11: not one of four)
    torch.cuda.synchronize()
    want = before.copy()
    for i in range(L):
        for kv in range(2):
            x = co.copy_pages(want[:, i, kv, :R, :, :d], [(4, 1, 9), (2, 3, 16)])
            want[:, i, kv, :R, :, :d] = co.keep_rows(x, table, rows, [[11, 3, 7, 0]], [4], [3])
    assert np.array_equal(read(flat), want)
    big = torch.zeros((5 << 30) // 2 + (1 << 20), device="cuda", dtype=torch.bfloat16)
    x, y = (z.as_strided((2, 16, 2, 64), (5 << 29, 128, 64, 1)) for z in (big, big[4096:]))
    x[0] = torch.randn(16, 2, 64, device="cuda").to(torch.bfloat16)
    far = lib.cache_layers([lib.paged_cache(x, y, put([[1, 0]]), put([20]))])
    lib.burst_attn_cache_copy_pages(far, put([[0, 1, 16]]))
    assert torch.equal(x[0], x[1])
    row = x[0, 3].clone()
    lib.burst_attn_cache_keep_rows(far, put([[19, 0]]), put([1]), new_rows=put([20]))              # (at most two tokens: 19 is none of them)
    assert torch.equal(x[0, 3], row) and torch.equal(x[0], x[1])
    last, first_new = x[0, 3].clone(), x[0, 2].clone()
    lib.burst_attn_cache_keep_rows(far, put([[1, 0]]), put([2]))                                   # rows 18 and 19 change places
    assert torch.equal(x[0, 2], last) and torch.equal(x[0, 3], first_new)


def test_captured_and_replayed(lib):
    """Both calls in a graph, replayed with other moves and lists between eager ones."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 92300))
    L, n_pages, R, Hkv, d, B, sq = 4, 30, 16, 2, 64, 3, 8
    dev, host = numbers(rng, L, n_pages, R, Hkv, d, False, True)
    table = rng.permutation(n_pages)[:B * 4].reshape(B, 4).astype(np.int32)
    layers = handles(lib, dev, table, [50, 64, 33])
    put = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    moves, source, kept = put([[0, 0, 0]] * 3), put(np.zeros((B, sq))), put([0] * B)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.burst_attn_cache_copy_pages(layers, moves)
        lib.burst_attn_cache_keep_rows(layers, source, kept)
    spare = [p for p in range(n_pages) if p not in table]
    for turn in range(4):
        m = [[int(table[turn % B, 0]), spare[turn], 16], [int(table[0, 2]), spare[turn + 5], 7], [1, 99, 3]]
        s, k = rng.integers(0, sq, (B, sq)), rng.integers(0, sq + 1, B)
        for x, y in ((moves, m), (source, s), (kept, k)):
            x.copy_(torch.from_numpy(np.asarray(y, np.int32)))
        graph.replay()
        host = [co.keep_rows(co.copy_pages(h, m), table, [50, 64, 33], s, [sq] * B, k) for h in host]
        torch.cuda.synchronize()
        for t, h in zip(dev, host):
            assert np.array_equal(read(t), h)
        lib.burst_attn_cache_keep_rows(layers, source, kept)
        host = [co.keep_rows(h, table, [50, 64, 33], s, [sq] * B, k) for h in host]
