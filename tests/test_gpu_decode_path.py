"""decode.py: a prompt through the ring's forward pass and into the devices' caches, then tokens one by one over all devices, against the
attention oracle over the whole sequence; and the handing out of pages."""
import math

import numpy as np
import pytest

from oracle import burst_oracle as oc
from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import helpers as hp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("partition,axes", [("zigzag", 1), ("striped", 3)])
def test_prompt_on_a_ring_then_tokens(lib, partition, axes):
    import torch
    from paper_2509_19836_amd import decode, ring
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 89000 + axes))
    B, Hq, Hkv, d, G, N, steps = 2, 8, 2, 64, 4, 512, 6
    scale, total = d ** -0.5, N + steps
    bits = {n: wl.f32_to_bf16_bits(rng.standard_normal((B, total, h, d), dtype=np.float32)) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
    dev, host = {n: hp.dev_bf16(b) for n, b in bits.items()}, {n: hp.widen(b) for n, b in bits.items()}
    freq = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    place = np.arange(total)
    pos = np.stack([place // 60, place // 6 % 10, place % 6])[:axes] if axes > 1 else place[None]
    pairs = [i % axes for i in range(d // 2)]
    f = torch.from_numpy(freq).cuda()
    rope_at = lambda rows: lib.rope(torch.from_numpy(np.repeat(pos[:, None, rows], B, 1).astype(np.int32)).cuda().contiguous(), f, axis_of_pair=pairs)
    rows = [hp.oracle_positions(oc, partition, g, G, N) for g in range(G)]
    caches, q_turned, k_turned, v_shards = [], [], [], []
    for g in range(G):
        cache = decode.PagedCache(2 * B + B * (N // G // 16 + 1), 16, B, Hkv, d, N // G + steps)
        n = rows[g].size
        part = {x: t[:, torch.from_numpy(rows[g]).cuda()].contiguous() for x, t in dev.items()}
        q_out = torch.empty_like(part["q"])
        cache.grow([n] * B)
        decode.append(cache, part["q"], part["k"], part["v"], rope_at(rows[g]), q_out)
        k_out = torch.empty_like(part["k"])
        lib.burst_attn_rope(lib.shape(B, Hq, Hkv, d, n, 0, 1.0), rope_at(rows[g]), part["q"], part["q"], part["k"], k_out)   # (q: not used again)
        caches.append(cache)
        q_turned.append(q_out)
        k_turned.append(k_out)
        v_shards.append(part["v"])
    bf16 = lambda x: hp.widen(wl.f32_to_bf16_bits(x.astype(np.float32)))
    kt = bf16(co.rope(host["k"], np.repeat(pos[:, None], B, 1), freq, pairs))
    qt = bf16(co.rope(host["q"], np.repeat(pos[:, None], B, 1), freq, pairs))
    # the prompt on device 1 of the ring
    i, n = 1, rows[1].size
    o_acc, lse_acc = torch.zeros(B, n, Hq, d, device="cuda"), torch.full((B, Hq, n), -math.inf, device="cuda")
    ring.ring_forward(i, G, N, partition, scale, q_turned[i], k_turned, v_shards, o_acc, lse_acc)
    vis = oc.visibility(rows[i], np.arange(N), True)
    O, L = oc.mha_attention_fwd(qt[:, rows[i]], kt[:, :N], host["v"][:, :N], scale, vis)
    assert hp.rel_err(o_acc.cpu().numpy(), O) <= hp.REL_TOL and hp.lse_err(lse_acc.cpu().numpy(), L) <= hp.LSE_TOL
    # tokens, dealt to the devices in turn
    q_out = torch.empty(B, 1, Hq, d, device="cuda", dtype=torch.bfloat16)
    o, o_part = (torch.empty(B, 1, Hq, d, device="cuda") for _ in range(2))
    lse, lse_part = (torch.empty(B, Hq, 1, device="cuda") for _ in range(2))
    ws = decode.workspace(caches[0], Hq)
    for s in range(steps):
        t, owner = N + s, s % G
        caches[owner].grow([1] * B)
        o.zero_()
        lse.fill_(-math.inf)
        one = {x: y[:, t:t + 1].contiguous() for x, y in dev.items()}
        decode.ring_token(caches, owner, one["q"], one["k"], one["v"], rope_at([t]), scale, q_out, o, lse, o_part, lse_part, ws)
        O, L = oc.mha_attention_fwd(qt[:, t:t + 1], kt[:, :t + 1], host["v"][:, :t + 1], scale)
        # turned numbers may fall on the other side of a rounding than the reference's: far inside the bar of the step
        assert hp.rel_err(o.cpu().numpy(), O) <= 2e-3 and hp.lse_err(lse.cpu().numpy(), L) <= hp.LSE_TOL


def test_pages_are_handed_out_and_come_back(lib):
    import torch
    from paper_2509_19836_amd import decode
    cache = decode.PagedCache(6, 16, 3, 1, 64, 64)
    cache.grow([17, 0, 16])
    assert cache.rows.tolist() == [17, 0, 16] and [len(p) for p in cache.pages] == [2, 0, 1]
    named = [cache.table[b, :len(p)].tolist() for b, p in enumerate(cache.pages)]
    assert named == cache.pages and len(set(sum(named, []))) == 3 and (cache.table >= 0).sum() == 3
    cache.grow([15, 0, 0])                                                 # fits in the second page
    assert [len(p) for p in cache.pages] == [2, 0, 1] and cache.rows.tolist() == [32, 0, 16]
    with pytest.raises(RuntimeError, match="pages"):
        cache.grow([17, 33, 0])                                            # 2 + 3 pages of 3
    with pytest.raises(ValueError, match="rows"):
        cache.grow([33, 0, 0])
    with pytest.raises(ValueError):
        cache.grow([1, 0])
    assert cache.rows.tolist() == [32, 0, 16] and len(cache.free) == 3
    cache.release(0)
    assert cache.rows.tolist() == [0, 0, 16] and len(cache.free) == 5 and (cache.table[0] == -1).all()
    cache.grow([0, 64, 16])
    assert sorted(sum(cache.pages, []) + cache.free) == list(range(6))
    x = torch.ones(3, 16, 1, 64, device="cuda", dtype=torch.bfloat16)
    decode.append(cache, x, x, x, lib.rope(torch.zeros(1, 3, 16, device="cuda", dtype=torch.int32), torch.ones(32, device="cuda")), torch.empty_like(x),
                  new_rows=torch.tensor([0, 0, 16], dtype=torch.int32, device="cuda"))
    k = cache.handle._tensors[0]
    assert (k[cache.pages[2][1]] == 1).all()
