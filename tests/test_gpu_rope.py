"""The rotation by positions on the GPU, element by element against the fp64 reference.

Tolerance of an element y = x1 c - x2 s: half a step of the result's type, relative to y (at a type's bottom, to its smallest normal number);
4 * 2^-24 of |x1| + |x2| for sine, cosine and three roundings in fp32 (each 2^-24 at most, the series 0.1 * 2^-24); and the angle's
own error, three roundings in 64 bits of the angle."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import helpers as hp

pytestmark = pytest.mark.gpu


def tolerance(x, y, angle, rotary_dim, adjacent, bf16):
    """Of each element of y, from x [batch, rows, heads, head_dim] and the angles [batch, rows, pairs]."""
    size = np.abs(np.asarray(x, np.float64))
    first, second = co.pair_elements(rotary_dim, adjacent)
    pair, off = np.zeros_like(size), np.zeros_like(size)
    both = size[..., first] + size[..., second]
    wrong = 3 * 2.0 ** -53 * np.abs(angle.astype(np.float64))[:, :, None] * both
    for side in (first, second):
        pair[..., side], off[..., side] = both, wrong
    return (2.0 ** -8 if bf16 else 2.0 ** -24) * np.maximum(np.abs(y), 2.0 ** -126) * (1 + 2.0 ** -7) + 4 * 2.0 ** -24 * pair + off


def _frequencies(pairs, base=10000.0):
    return (base ** (-np.arange(pairs) / pairs)).astype(np.float32)


CASES = [
    # batch, rows, q_heads, kv_heads, head_dim, rotary_dim, axes, adjacent, inverse, q and k in, q and k out
    (1, 1, 1, 1, 64, 64, 1, False, False, "bf16", "bf16"),
    (2, 3, 5, 1, 128, 128, 1, False, False, "bf16", "bf16"),
    (1, 77, 12, 12, 64, 32, 1, True, False, "bf16", "f32"),
    (3, 50, 7, 7, 128, 16, 2, False, True, "f32", "bf16"),
    (1, 257, 33, 3, 128, 112, 3, True, True, "f32", "f32"),
    (2, 129, 64, 8, 128, 128, 3, False, False, "bf16", "bf16"),
    (1, 300, 17, 17, 64, 48, 3, True, False, "bf16", "bf16"),
    (1, 5, 300, 2, 64, 64, 1, False, True, "f32", "f32"),
]


@pytest.mark.parametrize("case", CASES)
def test_against_the_reference(lib, case):
    import torch
    B, n, Hq, Hkv, d, R, axes, adjacent, inverse, x_type, y_type = case
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 81000 + n + Hq))
    pos = rng.integers(-1000, 200000, (axes, B, n)).astype(np.int32)
    pos[0, 0, 0], pos[-1, -1, -1] = 2 ** 31 - 1, -2 ** 31
    pairs = rng.integers(0, axes, R // 2).tolist()
    freq = _frequencies(R // 2)
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    host, dev, out, buffers = {}, {}, {}, {}
    for name, heads in (("q", Hq), ("k", Hkv)):
        x = rng.standard_normal((B, n, heads, d)).astype(np.float32)
        host[name] = hp.widen(wl.f32_to_bf16_bits(x)) if x_type == "bf16" else x.astype(np.float64)
        wide = torch.full((B, n + 2, heads + 1, d), float("nan"), device="cuda", dtype=types[x_type])     # strided, poison around it
        dev[name] = wide[:, 1:n + 1, :heads]
        dev[name].copy_(torch.from_numpy(host[name]))
        buffers[name] = torch.full((B, n + 1, heads + 2, d), 7.0, device="cuda", dtype=types[y_type])
        out[name] = buffers[name][:, :n, 1:heads + 1]
    r = lib.rope(torch.from_numpy(pos).cuda(), torch.from_numpy(freq).cuda(), adjacent=adjacent, axis_of_pair=pairs)
    print(f"rope {case}", flush=True)
    lib.burst_attn_rope(lib.shape(B, Hq, Hkv, d, n, 0, 1.0), r, dev["q"], out["q"], dev["k"], out["k"], inverse=inverse)
    torch.cuda.synchronize()
    angle = co.angles(pos, freq, pairs)
    for name in "qk":
        ref = co.rope(host[name], pos, freq, pairs, adjacent, inverse)
        got = out[name].double().cpu().numpy()
        assert (np.abs(got - ref) <= tolerance(host[name], ref, angle, R, adjacent, y_type == "bf16")).all()
        if x_type == y_type:
            assert np.array_equal(got[..., R:], host[name][..., R:])
        assert (buffers[name][:, n:] == 7).all() and (buffers[name][:, :, 0] == 7).all() and (buffers[name][:, :, -1] == 7).all()


def test_in_place_alone_and_there_and_back(lib):
    import torch
    B, n, H, d = 2, 65, 6, 128
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(B, n, H, d, generator=gen, device="cuda")
    pos = torch.arange(n, device="cuda", dtype=torch.int32).expand(1, B, n) * 1000     # (broadcast over the batch)
    r = lib.rope(pos, torch.from_numpy(_frequencies(d // 2)).cuda())
    shp = lib.shape(B, H, H, d, n, 0, 1.0)
    y = torch.empty_like(x)
    lib.burst_attn_rope(shp, r, x, y)                     # queries alone
    z = x.clone()
    lib.burst_attn_rope(shp, r, z, z)                     # in place: the same bits
    assert torch.equal(y, z)
    lib.burst_attn_rope(shp, r, z, z, inverse=True)
    # there and back: cos^2 + sin^2 = 1 and two rotations' roundings, 8 * 2^-24 of a pair's size each
    size = x.abs()[..., :d // 2] + x.abs()[..., d // 2:]
    assert ((z - x).abs() <= 16 * 2.0 ** -24 * torch.cat([size, size], -1)).all()


def test_gradient_of_the_backward_step(lib):
    """<turn(x), g> = <x, turn back(g)> for dQ as the backward step leaves it (fp32), and differences along one element."""
    import torch
    B, n, H, d = 1, 40, 3, 64
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, g = (torch.randn(B, n, H, d, generator=gen, device="cuda") for _ in range(2))
    pos = torch.stack([torch.arange(n, device="cuda") // 8, torch.arange(n, device="cuda") % 8]).to(torch.int32)[:, None].contiguous()
    r = lib.rope(pos, torch.from_numpy(_frequencies(16)).cuda(), adjacent=True, axis_of_pair=[0, 1] * 8)
    shp = lib.shape(B, H, H, d, n, 0, 1.0)
    y, dx, y2 = (torch.empty_like(x) for _ in range(3))
    lib.burst_attn_rope(shp, r, x, y, g, dx)              # (k: the wrong direction, overwritten below)
    lib.burst_attn_rope(shp, r, g, dx, inverse=True)
    left, right = (y.double() * g.double()).sum().item(), (x.double() * dx.double()).sum().item()
    scale = (x.double().abs() * g.double().abs()).sum().item()
    assert abs(left - right) <= 16 * 2.0 ** -24 * 2 * scale
    for at in ((0, 0, 0, 0), (0, 17, 1, 5), (0, 39, 2, 31), (0, 20, 0, 40)):
        x2 = x.clone()
        x2[at] += 1.0
        lib.burst_attn_rope(shp, r, x2, y2)
        slope = ((y2.double() - y.double()) * g.double()).sum().item() / (x2[at].double() - x[at].double()).item()
        assert abs(slope - dx[at].item()) <= 64 * 2.0 ** -24 * (x[at].abs().item() + 5.0) * g.abs().max().item()


def test_infinities_stay_in_their_pair(lib):
    import torch
    d = 64
    x = torch.ones(1, 1, 1, d, device="cuda", dtype=torch.bfloat16)
    x[..., 3], x[..., 40], x[..., 50] = float("inf"), float("nan"), float("-inf")
    r = lib.rope(torch.ones(1, 1, 1, device="cuda", dtype=torch.int32), torch.from_numpy(_frequencies(16)).cuda())
    y = torch.empty_like(x)
    lib.burst_attn_rope(lib.shape(1, 1, 1, d, 1, 0, 1.0), r, x, y)
    bad = (~torch.isfinite(y)).flatten().nonzero().flatten().tolist()
    assert bad == [3, 19, 40, 50] and y[0, 0, 0, 50] == float("-inf")


def test_no_rows(lib):
    import torch
    x = torch.zeros(1, 0, 2, 64, device="cuda", dtype=torch.bfloat16)
    r = lib.rope(torch.zeros(1, 1, 0, device="cuda", dtype=torch.int32), torch.ones(32, device="cuda"))
    if x.data_ptr() == 0:
        x = torch.zeros(1, 4, 2, 64, device="cuda", dtype=torch.bfloat16)
        with pytest.raises(ValueError):
            lib.burst_attn_rope(lib.shape(1, 2, 2, 64, 0, 0, 1.0), r, x, x)
        return
    lib.burst_attn_rope(lib.shape(1, 2, 2, 64, 0, 0, 1.0), r, x, x)


def test_far_strides_and_unaligned_plans(lib):
    """Rows more than 2^32 bytes apart in one tensor, and frequencies and positions that start at any 4 bytes."""
    import torch
    H, d, far = 2, 64, (1 << 32) + 4096
    flat = torch.zeros(far + 4 * H * d, device="cuda", dtype=torch.uint8).view(torch.bfloat16)
    x = flat.as_strided((2, 1, H, d), (far // 2, H * d, d, 1))
    rng = np.random.Generator(np.random.PCG64(9))
    bits = wl.f32_to_bf16_bits(rng.standard_normal((2, 1, H, d), dtype=np.float32))
    x.copy_(hp.dev_bf16(bits))
    freq, pos = _frequencies(32), np.array([3, 1000], np.int32)
    f = torch.zeros(33, device="cuda")[1:]
    f.copy_(torch.from_numpy(freq))
    p = torch.zeros(3, device="cuda", dtype=torch.int32)[1:].view(1, 2, 1)
    p.copy_(torch.from_numpy(pos).view(1, 2, 1))
    lib.burst_attn_rope(lib.shape(2, H, H, d, 1, 0, 1.0), lib.rope(p, f), x, x)
    host = hp.widen(bits)
    ref = co.rope(host, pos.reshape(1, 2, 1), freq, [0] * 32)
    angle = co.angles(pos.reshape(1, 2, 1), freq, [0] * 32)
    assert (np.abs(x.double().cpu().numpy() - ref) <= tolerance(host, ref, angle, d, False, True)).all()


@pytest.mark.parametrize("q_types,k_types", [(("f32", "bf16"), ("bf16", "f32")), (("bf16", "bf16"), ("f32", "f32"))])
def test_queries_and_keys_of_types_of_their_own(lib, q_types, k_types):
    """One launch for both, each tensor with its types: the bits of a launch for each."""
    import torch
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, Hq, Hkv, d = 33, 6, 2, 128
    x = {"q": torch.randn(1, n, Hq, d, generator=gen, device="cuda").to(types[q_types[0]]),
         "k": torch.randn(1, n, Hkv, d, generator=gen, device="cuda").to(types[k_types[0]])}
    empty = lambda name, to: torch.empty_like(x[name], dtype=types[to])
    together, alone = {"q": empty("q", q_types[1]), "k": empty("k", k_types[1])}, {"q": empty("q", q_types[1]), "k": empty("k", k_types[1])}
    r = lib.rope(torch.arange(n, device="cuda", dtype=torch.int32).view(1, 1, n), torch.from_numpy(_frequencies(48)).cuda(), adjacent=True)
    lib.burst_attn_rope(lib.shape(1, Hq, Hkv, d, n, 0, 1.0), r, x["q"], together["q"], x["k"], together["k"])
    lib.burst_attn_rope(lib.shape(1, Hq, Hq, d, n, 0, 1.0), r, x["q"], alone["q"])
    lib.burst_attn_rope(lib.shape(1, Hkv, Hkv, d, n, 0, 1.0), r, x["k"], alone["k"])
    assert torch.equal(together["q"], alone["q"]) and torch.equal(together["k"], alone["k"])


def test_captured_and_replayed(lib):
    """From one graph, with positions that the program changes between replays, and eager calls between: the eager bits every time."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(2, 5, 4, 64, generator=gen, device="cuda").to(torch.bfloat16)
    pos = torch.zeros(1, 2, 5, device="cuda", dtype=torch.int32)
    r, shp, y = lib.rope(pos, torch.from_numpy(_frequencies(32)).cuda()), lib.shape(2, 4, 4, 64, 5, 0, 1.0), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.burst_attn_rope(shp, r, x, y)
    for turn in range(4):
        pos += 1000 * turn + 1
        y.fill_(7.0)
        graph.replay()
        got = y.clone()
        lib.burst_attn_rope(shp, r, x, y)
        torch.cuda.synchronize()
        assert torch.equal(got, y) and not torch.equal(got, x)
