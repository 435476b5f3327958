"""decode.py: drafted words through two layers over one page table, scored, the right ones kept, against the same words one by one; sequences that begin with
another one's rows; a draft over the devices of a ring."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from oracle import lm_head_oracle as lmo
from paper_2509_19836_amd import workloads as wl
from tests import helpers as hp
from tests import test_gpu_tree as tt

pytestmark = pytest.mark.gpu


class Model:
    """Queries, keys and values of a layer are a word's own; the logits are products of what all layers' heads found."""
    def __init__(self, lib, rng, vocab, n_layers, Hq, Hkv, d):
        import torch
        table = lambda *sizes: hp.dev_bf16(wl.f32_to_bf16_bits(rng.standard_normal(sizes, dtype=np.float32)))
        self.lib, self.n_layers, self.scale = lib, n_layers, d ** -0.5
        self.q, self.k, self.v = (table(n_layers, vocab, h, d) for h in (Hq, Hkv, Hkv))
        self.out = table(vocab, Hq * d).float()
        self.freq = torch.from_numpy((10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)).cuda()

    def append(self, layers, words, positions, new_rows):
        """words [batch, n] into every layer's cache; the turned queries of each."""
        lib, turned = self.lib, []
        B, n = words.shape
        for i, layer in enumerate(layers):
            q, k, v = (x[i][words] for x in (self.q, self.k, self.v))
            out = q.clone()
            lib.burst_attn_cache_append(lib.shape(B, q.size(2), k.size(2), q.size(3), n, 0, 1.0), layer, k, v, new_rows, rope=lib.rope(positions, self.freq),
                                        q=q, q_out=out)
            turned.append(out)
        return turned

    def logits(self, found):
        B, n = found[0].shape[:2]
        return (sum(found).reshape(B * n, -1) @ self.out.T).contiguous()


def second_layer(lib, cache):
    import torch
    k, v = (torch.zeros_like(t) for t in cache.handle._tensors[:2])
    return [cache.handle, lib.paged_cache(k, v, cache.table, cache.rows)]


def rows_of(cache, layer, b):
    """Keys and values of a sequence, row after row."""
    import torch
    at = torch.tensor(cache.pages[b], device="cuda", dtype=torch.int64)
    return [t[at].flatten(0, 1)[:cache.lengths[b]].clone() for t in layer._tensors[:2]]


@pytest.mark.parametrize("window", [None, 9])
def test_drafted_words_are_the_words_one_by_one(lib, window):
    import torch
    from paper_2509_19836_amd import decode
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 97000 + (window or 0)))
    B, Hq, Hkv, d, vocab, most, page_rows, words_each = 3, 8, 2, 64, 499, 100, 16, 14
    model = Model(lib, rng, vocab, 2, Hq, Hkv, d)
    prompt, first = rng.integers(0, vocab, 21).tolist(), rng.integers(0, vocab, B).tolist()
    device = lambda x, dtype=torch.int64: torch.tensor(x, dtype=dtype, device="cuda")

    def begun():
        cache = decode.PagedCache(24, page_rows, B, Hkv, d, most)
        layers = second_layer(lib, cache)
        cache.grow([len(prompt), 0, 0])
        model.append(layers, device([prompt] * B), device([[range(len(prompt))]] , torch.int32).expand(1, B, -1), device([len(prompt), 0, 0], torch.int32))
        cache.fork(0, [1, 2], lib.cache_layers(layers))
        return cache, layers

    def seen_from(places):
        return None if window is None else device([max(0, t - window + 1) for t in places], torch.int32)

    # one by one
    plain, layers = begun()
    ws, truth = decode.workspace(plain, Hq), [[w] for w in first]
    lse = torch.empty(B, Hq, 1, device="cuda")
    for _ in range(words_each + 6):
        plain.grow([1] * B)
        places = [n - 1 for n in plain.lengths]
        turned = model.append(layers, device([[w[-1]] for w in truth]), device([[[t] for t in places]], torch.int32), device([1] * B, torch.int32))
        found = [torch.empty(B, 1, Hq, d, device="cuda") for _ in layers]
        for layer, q, o in zip(layers, turned, found):
            lib.burst_attn_decode(lib.shape(B, Hq, Hkv, d, 1, most, model.scale), layer, q, o, lse, ws, first_row=seen_from(places))
        for b, w in enumerate(model.logits(found).argmax(1).tolist()):
            truth[b].append(w)
    # drafts: the words that follow, as far as a guess is right, among wrong ones
    drafted, dlayers = begun()
    both = lib.cache_layers(dlayers)
    ws, said = decode.workspace(drafted, Hq, tokens=8), [[w] for w in first]
    plans = [([-1, 0, 0, 2, 2, 3], "+w++w+"), ([-1, 0, 1, 1], "++w+"), ([-1], "+"), ([-1, 0, 0, 0, 2, 4, 1, 6], "+wwwwwww"), ([-1, 0, 1, 2, 3], "+++++")]
    step = 0
    while min(map(len, said)) <= words_each:
        parents, kinds = zip(*(plans[(step + b) % len(plans)] for b in range(B)))
        guesses, expected = [], []
        for b in range(B):
            after, words, right = {}, [], []
            for i, (up, kind) in enumerate(zip(parents[b], kinds[b])):
                after[i] = 0 if up < 0 else after[up] + 1
                at = len(said[b]) - 1 + after[i]
                true = truth[b][at] if at < len(truth[b]) else 0
                good = kind == "+" and (up < 0 or up in right)
                right += [i] if good else []
                words.append(true if good else (true + 1 + i) % vocab)
            guesses.append(words)
            expected.append(right)
        held = list(drafted.lengths)
        draft = decode.Draft(drafted, parents, window=window)
        n = max(draft.counts)
        words = device([w + [0] * (n - len(w)) for w in guesses])
        turned = model.append(dlayers, words, draft.positions, draft.new_rows)
        found = [torch.zeros(B, n, Hq, d, device="cuda") for _ in dlayers]
        for layer, q, o in zip(dlayers, turned, found):
            lse = torch.zeros(B, Hq, n, device="cuda")
            decode.attend_tree(drafted, draft, q, model.scale, o, lse, ws, layer=layer)
            ref = co.tree(q.double().cpu().numpy(), *(t.double().cpu().numpy() for t in layer._tensors[:2]), drafted.table.cpu().numpy(), drafted.lengths,
                          draft.counts, model.scale, seen=[[sum(1 << j for j in range(i + 1) if continues(p, i, j, window)) for i in range(len(p))] for p in parents],
                          first=None if window is None else (draft.positions[0] - window + 1).cpu().numpy())
            shown = torch.where(torch.arange(n, device="cuda")[None, :, None, None] < draft.new_rows[:, None, None, None], o, 7.0)
            shown_lse = torch.where(torch.arange(n, device="cuda") < draft.new_rows[:, None, None], lse, 7.0)
            tt.check_tree(shown, shown_lse, ref, most, d)
        logits = model.logits(found)
        shp = lib.scores_shape(B * n, vocab, 2)
        top_logp, top_ids = torch.empty(B * n, 2, device="cuda"), torch.empty(B * n, 2, device="cuda", dtype=torch.int64)
        lib.burst_lm_head_scores(shp, logits, top_logp=top_logp, top_ids=top_ids,
                                 workspace=torch.empty(lib.burst_lm_head_scores_workspace_bytes(shp), device="cuda", dtype=torch.uint8))
        ref = lmo.scores(logits.double().cpu().numpy(), n_top=2)          # (off by at most (5 * 100 + 499 + 8 + 200) 2^-24 = 7.2e-5 with logits up to 100)
        assert (top_ids.cpu().numpy() == ref["top_ids"]).all() and np.abs(top_logp.cpu().numpy() - ref["top_logp"]).max() <= 1e-4
        likeliest = top_ids[:, 0].reshape(B, n).tolist()
        paths = draft.agreed(guesses, likeliest)
        assert paths == expected
        drafted.keep(draft.counts, paths, both)
        assert drafted.lengths == [h + len(p) for h, p in zip(held, paths)] and drafted.rows.tolist() == drafted.lengths
        for b, path in enumerate(paths):
            said[b] += [guesses[b][i] for i in path[1:]] + [likeliest[b][path[-1]]]
            assert said[b] == truth[b][:len(said[b])]
        step += 1
    for b in range(B):
        for layer, other in zip(layers, dlayers):
            for x, y in zip(rows_of(drafted, other, b), rows_of(plain, layer, b)):
                assert x.view(torch.int16).equal(y[:x.size(0)].view(torch.int16))
        assert len(drafted.pages[b]) == -(-drafted.lengths[b] // page_rows) and (drafted.table[b] >= 0).sum() == len(drafted.pages[b])
    assert sorted(set(sum(drafted.pages, []) + drafted.free)) == list(range(24)) and drafted.holders[drafted.pages[0][0]] == 3


def continues(parents, i, j, window):
    """Whether token i continues token j (or is it), with fewer than `window` tokens from one to the other."""
    far = 0
    while i > j:
        i, far = parents[i], far + 1
    return i == j and (window is None or far < window)


def test_sequences_that_begin_alike(lib):
    import torch
    from paper_2509_19836_amd import decode
    B, Hkv, d, page_rows = 4, 2, 64, 16
    cache = decode.PagedCache(9, page_rows, B, Hkv, d, 64)
    layers = second_layer(lib, cache)
    both = lib.cache_layers(layers)
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 97100))

    def append(counts):
        n = max(counts)
        x = [[hp.dev_bf16(wl.f32_to_bf16_bits(rng.standard_normal((B, n, Hkv, d), dtype=np.float32))) for _ in "kv"] for _ in layers]
        for layer, (k, v) in zip(layers, x):
            lib.burst_attn_cache_append(lib.shape(B, Hkv, Hkv, d, n, 0, 1.0), layer, k, v, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        return x
    cache.grow([37, 0, 0, 5])
    append([37, 0, 0, 5])
    cache.fork(0, [1, 2], both)
    assert cache.lengths == [37, 37, 37, 5] and cache.rows.tolist() == cache.lengths
    assert cache.pages[0][:2] == cache.pages[1][:2] == cache.pages[2][:2] and len({cache.pages[b][2] for b in range(3)}) == 3 and len(cache.free) == 3
    before = [[rows_of(cache, layer, 0) for layer in layers]] * 3
    cache.grow([3, 1, 12, 0])
    fresh = append([3, 1, 12, 0])
    for b, n in enumerate([3, 1, 12]):
        for i, layer in enumerate(layers):
            for x, old, new in zip(rows_of(cache, layer, b), before[b][i], fresh[i]):
                assert x.equal(torch.cat([old, new[b, :n]]))
    assert len(cache.free) == 2                                               # sequence 2 has gone on into another page
    kept = (list(cache.lengths), [list(p) for p in cache.pages], list(cache.free), list(cache.holders), cache.table.clone())
    for call, error in ((lambda: cache.fork(0, [1]), ValueError), (lambda: cache.fork(3, [3]), ValueError), (lambda: cache.fork(3, [-1]), ValueError), (lambda: cache.fork(-1, []), ValueError), (lambda: cache.keep([9, 0, 0, 0], [[0], [], [], []]), ValueError),
                        (lambda: cache.keep([2, 0, 0, 0], [[2], [], [], []]), ValueError), (lambda: cache.keep([2, 0, 0], [[0], [], []]), ValueError),
                        (lambda: cache.keep([0, 0, 0, 6], [[], [], [], [0]]), ValueError), (lambda: decode.Draft(cache, [[0], [], [], []]), ValueError),
                        (lambda: decode.Draft(cache, [[], [], [], []]), ValueError), (lambda: decode.Draft(cache, [[-1] * 60, [], [], []]), ValueError)):
        with pytest.raises(error):
            call()
    assert kept[:4] == (cache.lengths, cache.pages, cache.free, cache.holders) and kept[4].equal(cache.table) and cache.rows.tolist() == cache.lengths
    cache.keep([0, 1, 12, 0], [[], [], [11, 3], []], both)
    assert cache.lengths == [40, 37, 39, 5] and len(cache.free) == 3
    for i, layer in enumerate(layers):
        for x, old, new in zip(rows_of(cache, layer, 2), before[2][i], fresh[i]):
            assert x.equal(torch.cat([old, new[2, [11, 3]]]))
    shared = cache.pages[0][0]
    for b, left in ((0, 2), (2, 1)):
        cache.release(b)
        assert cache.holders[shared] == left and shared not in cache.free
    cache.release(1)
    cache.release(3)
    assert sorted(cache.free) == list(range(9)) and cache.holders == [0] * 9
    cache.grow([32, 0, 0, 0])
    cache.fork(0, [1, 2, 3])                                                  # nothing but full pages
    assert len(cache.free) == 7 and cache.pages[1] == cache.pages[0]
    cache.grow([1, 1, 1, 1])
    with pytest.raises(RuntimeError, match="pages"):
        cache.grow([16] * 4)


def test_a_draft_over_a_ring(lib):
    import torch
    from paper_2509_19836_amd import decode
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 97200))
    B, Hq, Hkv, d, G = 2, 8, 2, 64, 3
    scale = d ** -0.5
    rows = [[20, 31], [0, 17], [25, 8]]                                       # of each device, of each sequence
    parents = [[-1, 0, 0, 1, 1, 4, -1], [-1, 0, 1, 2, 3]]
    caches, held = [], [[], []]
    x = lambda *sizes: hp.dev_bf16(wl.f32_to_bf16_bits(rng.standard_normal(sizes, dtype=np.float32)))
    for g in range(G):
        cache = decode.PagedCache(8, 16, B, Hkv, d, 64)
        cache.grow(rows[g])
        k, v = x(B, max(rows[g]), Hkv, d), x(B, max(rows[g]), Hkv, d)
        lib.burst_attn_cache_append(lib.shape(B, Hkv, Hkv, d, max(rows[g]), 0, 1.0), cache.handle, k, v, torch.tensor(rows[g], dtype=torch.int32, device="cuda"))
        for b in range(B):
            held[b].append([t[b, :rows[g][b]].double().cpu().numpy() for t in (k, v)])
        caches.append(cache)
    owner, after = 1, [sum(r[b] for r in rows) for b in range(B)]
    with pytest.raises(ValueError, match="window"):
        decode.Draft(caches[owner], parents, window=5, after=after)
    with pytest.raises(ValueError):
        decode.Draft(caches[owner], parents, after=after[:1])
    assert caches[owner].lengths == rows[owner]
    draft = decode.Draft(caches[owner], parents, after=after)
    assert draft.positions.tolist() == [[[45, 46, 46, 47, 47, 48, 45], [56, 57, 58, 59, 60, 56, 56]]]
    n = 7
    q, k, v = x(B, n, Hq, d), x(B, n, Hkv, d), x(B, n, Hkv, d)
    rope = lib.rope(draft.positions, torch.zeros(d // 2, device="cuda"))      # (turned by nothing, so that the oracle has the very numbers)
    q_out = torch.empty_like(q)
    o, lse = torch.zeros(B, n, Hq, d, device="cuda"), torch.full((B, Hq, n), -math.inf, device="cuda")
    o_part, lse_part = torch.zeros_like(o), torch.zeros_like(lse)
    ws = decode.workspace(caches[0], Hq, tokens=n)
    decode.ring_draft(caches, owner, draft, q, k, v, rope, scale, q_out, o, lse, o_part, lse_part, ws)
    for b in range(B):
        count = draft.counts[b]
        K, V = (np.concatenate([part[i] for part in held[b]] + [t[b, :count].double().cpu().numpy()]) for i, t in ((0, k), (1, v)))
        seen = [[sum(1 << j for j in range(i + 1) if continues(parents[b], i, j, None)) for i in range(count)]]
        ref = co.tree(q[b:b + 1].double().cpu().numpy(), K[None], V[None], np.zeros((1, 1), np.int32), [K.shape[0]], [count], scale, seen=seen)
        tt.check_tree(torch.where(torch.arange(n, device="cuda")[:, None, None] < count, o[b:b + 1], 7.0),
                      torch.where(torch.arange(n, device="cuda") < count, lse[b:b + 1], 7.0), ref, 64, d)
