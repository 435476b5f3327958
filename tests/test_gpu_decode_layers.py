"""Two layers of a model over one page table: a second layer's pages in tensors of its own, by the table and the numbers of rows of the first's cache."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import helpers as hp
from tests import test_gpu_paged_cache as tp

pytestmark = pytest.mark.gpu


def test_two_layers_over_one_table(lib):
    import torch
    from paper_2509_19836_amd import decode
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 91000))
    B, Hq, Hkv, d, page_rows, most = 3, 6, 2, 64, 16, 100
    cache = decode.PagedCache(20, page_rows, B, Hkv, d, most)
    k2, v2 = (torch.empty(20, page_rows, Hkv, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))     # (in another order of memory)
    layers = [cache.handle, lib.paged_cache(k2, v2, cache.table, cache.rows)]
    held = [{x: [np.zeros((0, Hkv, d))] * B for x in "kv"} for _ in layers]
    ws = decode.workspace(cache, Hq)
    for counts in ([40, 1, 17], [1, 1, 1], [1, 0, 1], [20, 30, 0], [1, 1, 1]):
        cache.grow(counts)                                                  # once for both layers
        n, new = max(counts), torch.tensor(counts, dtype=torch.int32, device="cuda")
        for layer, have in zip(layers, held):
            bits = {x: wl.f32_to_bf16_bits(rng.standard_normal((B, n, Hkv, d), dtype=np.float32)) for x in "kv"}
            lib.burst_attn_cache_append(lib.shape(B, Hq, Hkv, d, n, 0, 1.0), layer, hp.dev_bf16(bits["k"]), hp.dev_bf16(bits["v"]), new)
            for x in "kv":
                have[x] = [np.concatenate([have[x][b], hp.widen(bits[x])[b, :counts[b]]]) for b in range(B)]
            q, q_host = tp.queries(rng, B, Hq, d)
            o, lse = torch.empty(B, 1, Hq, d, device="cuda"), torch.empty(B, Hq, 1, device="cuda")
            lib.burst_attn_decode(lib.shape(B, Hq, Hkv, d, 1, most, d ** -0.5), layer, q, o, lse, ws)
            for b in range(B):                                              # each sequence as one page
                ref = co.decode(q_host[b:b + 1], have["k"][b][None], have["v"][b][None], np.zeros((1, 1), np.int32), [cache.lengths[b]], d ** -0.5)
                tp.check_decode(o[b:b + 1], lse[b:b + 1], ref, most, d)
