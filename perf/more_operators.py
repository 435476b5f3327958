"""Attention of drafted tokens over a paged cache, pages and rows of a cache copied, and scores of tokens, as measurable cases.

A case is a dict of plain values:

  op "tree"    attention of a few new tokens of every sequence over its rows in the cache: each sees its ancestors among the new ones, and of the
               older rows all, or a window and a few first ones.
  op "copy"    the first rows of pages copied to other pages, in all layers of a model.
  op "keep"    of the new rows those that were accepted, moved to the front, in all layers.
  op "step"    what a layer does when drafts are checked: append, attention, and, once they are accepted, the rows that stay.
  op "scores"  log probability of given tokens, log-sum-exp, entropy and the likeliest words from logits.
  op "train"   the same without the likeliest words, then the gradient of the logits.

batch: sequences; new: tokens that a sequence brings (at most; where "ragged" is set some bring fewer); rows: the longest sequence's rows in the
cache, the new ones among them.
"""
import math
import random

import torch

own = False     # whether run() makes the library's calls or computes the plain form

MAX_BYTES, MAX_FLOPS = 2.1e9, 2.7e11      # of a drawn case's pass: just under the largest listed ones
F8_MAX = 448.0                            # the largest e4m3 number


def _case(name, op, **kw):
    case = dict(name=name, op=op)
    if op in ("scores", "train"):
        case.update(tokens=64, vocab=32000, logits="bf16", scale=1.0, allowed=1.0, n_top=8 if op == "scores" else 0)
    else:
        case.update(batch=1, q_heads=32, kv_heads=8, head_dim=128, new=8, rows=4096, ragged=False, page_rows=64, cache="bf16", by_head=False)
        if op in ("tree", "step"):
            case.update(chain=False, window=0, sinks=0, elsewhere=False, o="bf16")
        if op in ("copy", "keep"):
            case.update(layers=1)
        if op == "copy":
            case.update(pages=8)
    case.update(kw)
    return case


def listed():
    return [
        # one user of a small model with 64-wide heads whose next five tokens were guessed, a length that fits no tile and no page
        _case("tree_one_short", "tree", q_heads=12, kv_heads=12, head_dim=64, new=5, rows=777, page_rows=16, chain=True),
        # wide trees of drafts over long contexts: products count as much as the cache
        _case("tree_wide_b4", "tree", batch=4, q_heads=64, new=64, rows=32768, by_head=True),
        # many users, a cache of 8 bits, a window and the first tokens
        _case("tree_window_f8_b32", "tree", batch=32, q_heads=64, new=8, rows=49152, ragged=True, cache="f8", window=16384, sinks=4),
        # one device's share of a 1M-token sequence over 8 devices; the drafts' own rows are another device's
        _case("tree_1m_share", "tree", q_heads=32, kv_heads=32, new=4, rows=131072, page_rows=256, by_head=True, elsewhere=True, o="f32"),
        # a layer's work when the drafts of many chats are checked
        _case("step_chats_b16", "step", batch=16, new=12, rows=4096, ragged=True, page_rows=16),
        # four continuations of one prompt: its last page once more for each
        _case("copy_last_pages", "copy", rows=2000, pages=3, page_rows=64, layers=2, by_head=True),
        # pages moved together, all layers of a model
        _case("copy_pages_layers", "copy", q_heads=8, pages=64, rows=8192, layers=32, page_rows=64),
        # accepted drafts of many chats, all layers of a model
        _case("keep_b32_layers", "keep", batch=32, new=16, rows=1024, ragged=True, layers=32, page_rows=16),
        # the drafts of a few chats under the model that checks them
        _case("scores_verify", "scores", tokens=60),
        # every token of a long prompt, with alternatives
        _case("scores_prompt", "scores", tokens=4001, vocab=128256, n_top=20),
        # a batch of answers with their advantages, logits in 32 bits
        _case("train_answers_f32", "train", tokens=4096, logits="f32"),
        # a short odd batch with a vocabulary that fits nothing, sampled at a temperature, words forbidden by a grammar
        _case("train_odd_masked", "train", tokens=331, vocab=50257, scale=1.25, allowed=0.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["tree", "tree", "tree", "step", "copy", "keep", "scores", "train"])
        if op in ("scores", "train"):
            kw = dict(tokens=_log_int(rng, 1, 16384), vocab=_log_int(rng, 200, 262144), logits=rng.choice(["bf16", "f32"]),
                      scale=rng.choice([1.0, 1.0, 0.7, 1.6]), allowed=rng.choice([1.0, 1.0, 0.5, 0.02]))
            if op == "scores":
                kw["n_top"] = rng.choice([0, 1, 4, 8, 20, 32, 64])
        else:
            kv = rng.choice([1, 2, 4, 5, 8, 12, 16, 32])
            group = rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16, 32) if kv * g <= 64])
            kw = dict(batch=rng.choice([1, 1, 2, 3, 7, 8, 16, 32, 64, 128]), q_heads=kv * group, kv_heads=kv, head_dim=rng.choice([64, 128, 128]),
                      new=_log_int(rng, 1, 64), page_rows=rng.choice([1, 16, 16, 32, 48, 64, 128, 256]), cache=rng.choice(["bf16", "bf16", "f8"]),
                      by_head=rng.random() < 0.4)
            kw["rows"] = max(kw["new"], _log_int(rng, 1, 262144 if op in ("tree", "step") else 4096))
            kw["ragged"] = kw["batch"] > 1 and rng.random() < 0.7
            if op in ("tree", "step"):
                kw.update(chain=rng.random() < 0.3, o=rng.choice(["bf16", "f32"]), elsewhere=op == "tree" and rng.random() < 0.15)
                if rng.random() < 0.3:
                    kw.update(window=_log_int(rng, 1, kw["rows"]), sinks=rng.choice([0, 1, 4, 64, 100]))
            else:
                kw["layers"] = _log_int(rng, 1, 48)
            if op == "copy":
                kw.update(batch=1, ragged=False, pages=_log_int(rng, 1, 512))
        case = _case("", op, **kw)
        del case["name"]
        w = work(case)
        # what a pass moves, the plain form's copies of the cache in 32 bits, padded to the longest sequence, and its scores
        cells = state = 0
        if op in ("tree", "step"):
            cells = case["batch"] * case["rows"] * max(case["kv_heads"] * case["head_dim"], case["q_heads"] * case["new"])
        if op in ("copy", "keep"):
            state = case["layers"] * (_pages(case) + 1) * case["page_rows"] * case["kv_heads"] * case["head_dim"]
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS and cells <= 1.1e9 and state <= 6e8:
            return case


# ---- what a case says about its sequences ----------------------------------------------------------------

def _spread(case, most, least, salt):
    """Lengths of the case's sequences: the longest first, the others spread over the logarithm of the range."""
    if not case["ragged"]:
        return [most] * case["batch"]
    rng = random.Random(salt * 1000003 + most * 131 + case["batch"])
    return [most] + [max(least, min(most, _log_int(rng, max(least, most // 20), most))) for _ in range(case["batch"] - 1)]


def _new(case):
    return _spread(case, case["new"], 1, 1)


def _rows(case):
    """Rows in the cache, the new ones among them."""
    return [max(n, r) for n, r in zip(_new(case), _spread(case, case["rows"], 1, 2))]


def _pages(case):
    """Pages that sequences have (copy: those to be copied, the pages they go to, and the sequences' other ones)."""
    if case["op"] == "copy":
        return 2 * case["pages"] + -(-case["rows"] // case["page_rows"])
    return sum(-(-r // case["page_rows"]) for r in _rows(case))


def _parents(case):
    """For each sequence the parent of every new token, an earlier one or -1: a chain, or a tree that thins out as it grows."""
    if case["chain"]:
        return [[i - 1 for i in range(n)] for n in _new(case)]
    rng = random.Random(case["new"] * 7919 + case["batch"])
    return [[rng.randrange(max(-1, i - 6), i) for i in range(n)] for n in _new(case)]


def _seen_words(parents):
    """Bit j of word i: token i sees new token j, its ancestors and itself."""
    words = []
    for i, p in enumerate(parents):
        words.append((words[p] if p >= 0 else 0) | 1 << i)
    return words


def _first_rows(case):
    """For each sequence and token the first older row of its window."""
    first = []
    for rows, parents in zip(_rows(case), _parents(case)):
        older = rows if case["elsewhere"] else rows - len(parents)
        depth = []
        for p in parents:
            depth.append(depth[p] + 1 if p >= 0 else 0)
        first.append([max(0, older + k - case["window"] + 1) if case["window"] else 0 for k in depth])
    return first


def _kept(case):
    """For each sequence the new tokens that were accepted: a path from the front of the tree on."""
    rng = random.Random(case["new"] * 104729 + case["batch"])
    kept = []
    for n in _new(case):
        path, i = [], rng.randrange(min(n, 2))
        while i < n:
            path.append(i)
            i += rng.randrange(1, 5)
        kept.append(path[:rng.randrange(1, len(path) + 1)])
    return kept


# ---- inputs ----------------------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _padded(lists, width, fill, dtype):
    return torch.tensor([x + [fill] * (width - len(x)) for x in lists], dtype=dtype, device="cuda")


def _signed(word):
    return word - (1 << 64) if word >> 63 else word


def _cache_inputs(case, gen, s):
    n_layers, Hkv, d, R = case.get("layers", 1), case["kv_heads"], case["head_dim"], case["page_rows"]
    f8, n_pages = case["cache"] == "f8", _pages(case) + 1
    shape = (n_layers, n_pages, Hkv, R, d) if case["by_head"] else (n_layers, n_pages, R, Hkv, d)
    for name in ("K", "V"):
        x = torch.empty(shape, device="cuda", dtype=torch.float8_e4m3fn if f8 else torch.bfloat16)
        flat = x.view(n_layers * n_pages, *shape[2:])
        each = max(1, (1 << 26) // (R * Hkv * d))
        for i in range(0, flat.size(0), each):                       # keys and values of unit size, in 8 bits over a scale of their head
            part = torch.randn(flat[i:i + each].shape, generator=gen, device="cuda")
            flat[i:i + each] = (part * 96.0).clamp(-F8_MAX, F8_MAX).to(x.dtype) if f8 else part.to(x.dtype)
        s[name] = x.transpose(2, 3) if case["by_head"] else x        # [layers, pages, rows, heads, head_dim]
        s[name + "_scale"] = (0.75 + 0.5 * torch.rand(Hkv, generator=gen, device="cuda")) / 96.0 if f8 else None
    return n_pages


def _prepare_cache(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, n, Hq, Hkv, d, R = case["batch"], case["new"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page_rows"]
    s = {"case": case}
    n_pages = _cache_inputs(case, gen, s)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32).tolist()
    rows, new = _rows(case), _new(case)
    pages = [-(-r // R) for r in rows]
    table, at = [], 0
    for p in pages:
        table.append(order[at:at + p])
        at += p
    s.update(table=_padded(table, max(pages) + 1, 0, torch.int32), rows=torch.tensor(rows, dtype=torch.int32, device="cuda"),
             tokens=torch.tensor(new, dtype=torch.int32, device="cuda"), max_rows=max(rows), scale=d ** -0.5)
    if case["op"] == "copy":
        n_copies = case["pages"]
        # whole pages, and for a fork the rows that the sequence has of its last page
        part = [R if n_copies > 4 else max(1, case["rows"] % R)] * n_copies
        source = order[at:at + n_copies] if n_copies > 4 else [order[at - 1]] * n_copies
        s["moves"] = torch.tensor([list(m) for m in zip(source, order[at + n_copies:at + 2 * n_copies], part)], dtype=torch.int32, device="cuda")
    if case["op"] in ("keep", "step"):
        kept = _kept(case)
        s["from"] = _padded(kept, n, 0, torch.int32)
        s["kept"] = torch.tensor([len(k) for k in kept], dtype=torch.int32, device="cuda")
    if case["op"] in ("tree", "step"):
        s["q"] = torch.randn(B, n, Hq, d, generator=gen, device="cuda").to(torch.bfloat16)
        s["o"] = torch.zeros(B, n, Hq, d, device="cuda", dtype=_TYPES[case["o"]])          # padding stays as it is
        s["lse"] = torch.zeros(B, Hq, n, device="cuda")
        words = [_seen_words(p) for p in _parents(case)]
        s["seen"] = _padded([[_signed(w) for w in x] for x in words], n, 0, torch.int64)
        s["first"] = _padded(_first_rows(case), n, 0, torch.int32)
    if case["op"] == "step":
        s["k"], s["v"] = (torch.randn(B, n, Hkv, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    return s


def _prepare_scores(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, v = case["tokens"], case["vocab"]
    x = torch.empty(n, v, device="cuda", dtype=_TYPES[case["logits"]])
    each = max(1, (1 << 27) // v)
    for i in range(0, n, each):                                      # a few likely words above many unlikely ones
        part = torch.randn(x[i:i + each].shape, generator=gen, device="cuda")
        part = 2.0 * part + 0.5 * part.abs() * part
        if case["allowed"] < 1.0:
            part.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") >= case["allowed"], -math.inf)
            part[:, v // 2] = 0.0                                    # (no grammar forbids everything)
        x[i:i + each] = part
    y = torch.randint(0, v, (n,), generator=gen, device="cuda")
    y[torch.rand(n, generator=gen, device="cuda") < 0.05] = -1       # padding between answers
    s = {"case": case, "logits": x, "y": y}
    f32 = dict(device="cuda", dtype=torch.float32)
    s["logp"], s["lse"], s["entropy"] = (torch.empty(n, **f32) for _ in range(3))
    if case["op"] == "scores":
        s["top_logp"], s["top_ids"] = torch.empty(n, case["n_top"], **f32), torch.empty(n, case["n_top"], device="cuda", dtype=torch.int64)
    else:
        s["g_logp"] = torch.randn(n, generator=gen, **f32) / n       # advantages
        s["g_entropy"] = torch.full((n,), -0.01 / n, **f32)          # a reward for entropy
        s["g_lse"] = 1e-3 * torch.rand(n, generator=gen, **f32) / n  # a penalty on the size of the logits
        s["d_logits"] = torch.empty_like(x)
    return s


def _descriptors(s):
    """What a user of the library fills in once, for a layer and its buffers, and keeps: sizes, the caches, the tree, workspaces."""
    from paper_2509_19836_amd import binding as lib
    case = s["case"]
    if case["op"] in ("scores", "train"):
        s["shape"] = lib.scores_shape(case["tokens"], case["vocab"], case["n_top"], case["scale"])
        s["ws"] = torch.empty(lib.burst_lm_head_scores_workspace_bytes(s["shape"]), device="cuda", dtype=torch.uint8)
        return
    caches = [lib.paged_cache(k, v, s["table"], s["rows"], k_scale=s["K_scale"], v_scale=s["V_scale"]) for k, v in zip(s["K"], s["V"])]
    s["cache"], s["layers"] = caches[0], lib.cache_layers(caches)
    if case["op"] in ("tree", "step"):
        sizes = [case[name] for name in ("batch", "q_heads", "kv_heads", "head_dim")]
        s["shape"] = lib.shape(*sizes, case["new"], s["max_rows"], s["scale"])
        s["tree"] = lib.tree(seen=None if case["chain"] else s["seen"], first_row=s["first"] if case["window"] else None, tokens=s["tokens"],
                             sink_rows=case["sinks"], elsewhere=case["elsewhere"])
        s["ws"] = torch.empty(lib.burst_attn_tree_workspace_bytes(s["shape"]), device="cuda", dtype=torch.uint8)


def prepare(case, seed):
    s = (_prepare_scores if case["op"] in ("scores", "train") else _prepare_cache)(case, seed)
    if own:
        _descriptors(s)
    return s


# ---- the plain form --------------------------------------------------------------------------------------

def _bytes(s, name):
    """The cache as numbers that may be indexed: e4m3 as its bytes."""
    return s[name].view(torch.uint8) if s["case"]["cache"] == "f8" else s[name]


def _new_places(s, i):
    """Page, and row in it, of the sequences' new tokens i [batch, n]."""
    R, row = s["case"]["page_rows"], (s["rows"] - s["tokens"]).long()[:, None] + i
    return torch.gather(s["table"].long(), 1, row // R), row % R


def _plain_append(s):
    case = s["case"]
    i = torch.arange(case["new"], device="cuda")
    i = torch.minimum(i[None].expand(case["batch"], -1), (s["tokens"] - 1)[:, None].long())      # padding puts the last row once more
    page, r = _new_places(s, i)
    for name, x in (("K", s["k"]), ("V", s["v"])):
        x = torch.gather(x.float(), 1, i[:, :, None, None].expand_as(x))
        if case["cache"] == "f8":
            x = (x / s[name + "_scale"][:, None]).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        _bytes(s, name)[0][page, r] = x.to(_bytes(s, name).dtype)


def _gathered(s, name):
    """Keys or values of all sequences, [batch, kv_heads, rows, head_dim] in 32 bits, padded to the longest."""
    case, cols = s["case"], -(-s["max_rows"] // s["case"]["page_rows"])
    x = _bytes(s, name)[0][s["table"][:, :cols].long()]
    x = x.view(torch.float8_e4m3fn) if case["cache"] == "f8" else x
    x = x.flatten(1, 2)[:, :s["max_rows"]].permute(0, 2, 1, 3).float()
    return x * s[name + "_scale"][:, None, None] if case["cache"] == "f8" else x


def _plain_tree(s):
    case = s["case"]
    B, n, Hq, Hkv, d = case["batch"], case["new"], case["q_heads"], case["kv_heads"], case["head_dim"]
    q = s["q"].float().view(B, n, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)       # columns: (head of the group, token)
    score = torch.matmul(q, _gathered(s, "K").transpose(2, 3)).mul_(s["scale"])
    t = torch.arange(s["max_rows"], device="cuda")
    older = s["rows"] if case["elsewhere"] else s["rows"] - s["tokens"]
    j = t[None] - older[:, None]                                                                         # [batch, rows]: which new token
    seen = ((t[None, None] >= s["first"][:, :, None]) | (t < case["sinks"])[None, None]) & (j < 0)[:, None]
    among = (s["seen"][:, :, None] >> j.clamp(0, 63)[:, None]) & 1
    seen |= (among != 0) & (j >= 0)[:, None]
    seen &= (t[None] < s["rows"][:, None])[:, None]
    score = score.view(B, Hkv, -1, n, s["max_rows"]).masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, s["max_rows"]), _gathered(s, "V")).view(B, Hkv, -1, n, d) / torch.where(total == 0, 1.0, total)
    valid = torch.arange(n, device="cuda")[None] < s["tokens"][:, None]
    s["o"].copy_(torch.where(valid[:, :, None, None], o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, d).to(s["o"].dtype), s["o"]))
    s["lse"].copy_(torch.where(valid[:, None], (top + torch.log(total)).reshape(B, Hq, n), s["lse"]))
    return [s["o"], s["lse"]]


def _plain_copy(s):
    source, to, part = s["moves"].long().unbind(1)
    r = torch.arange(s["case"]["page_rows"], device="cuda")
    for name in ("K", "V"):
        x = _bytes(s, name)
        x[:, to] = torch.where((r[None] < part[:, None])[None, :, :, None, None], x[:, source], x[:, to])
    return [s["K"], s["V"]]


def _plain_keep(s):
    case = s["case"]
    i = torch.arange(case["new"], device="cuda")[None].expand(case["batch"], -1)
    stays = i < s["kept"][:, None]
    page, r = _new_places(s, torch.where(stays, s["from"].long(), torch.minimum(i, (s["tokens"] - 1)[:, None].long())))
    to_page, to_r = _new_places(s, torch.minimum(i, (s["tokens"] - 1)[:, None].long()))
    for name in ("K", "V"):
        x = _bytes(s, name)
        x[:, to_page[stays], to_r[stays]] = x[:, page[stays], r[stays]]
    return [s["K"], s["V"]]


def _plain_scores(s):
    case = s["case"]
    raw = s["logits"].float()
    x = raw * case["scale"]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    s["lse"].copy_((top + torch.log(total))[:, 0])
    s["entropy"].copy_((torch.log(total) - (e * torch.where(e == 0, 0.0, x - top)).sum(1, keepdim=True) / total)[:, 0])
    at = torch.gather(x, 1, s["y"].clamp(min=0)[:, None])[:, 0]
    s["logp"].copy_(torch.where(s["y"] >= 0, at - s["lse"], 0.0))
    out = [s["logp"], s["lse"], s["entropy"]]
    if case["op"] == "scores" and case["n_top"] > 0:
        # the order of the numbers as that of whole ones, the lowest index first among equals
        bits = raw.view(torch.int32).long()
        key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * (1 << 31) + (case["vocab"] - 1 - torch.arange(case["vocab"], device="cuda"))
        ids = torch.topk(key, case["n_top"], dim=1).indices
        s["top_ids"].copy_(ids)
        s["top_logp"].copy_(torch.gather(x, 1, ids) - s["lse"][:, None])
        out += [s["top_logp"], s["top_ids"]]
    return out


def _plain_train(s):
    case, out = s["case"], _plain_scores(s)
    logp = s["logits"].float() * case["scale"] - s["lse"][:, None]
    p = torch.exp(logp)
    by_entropy = s["g_entropy"][:, None] * (torch.where(p == 0, 0.0, logp) + s["entropy"][:, None])
    g_logp = torch.where(s["y"] >= 0, s["g_logp"], 0.0)
    g = p * ((s["g_lse"] - g_logp)[:, None] - by_entropy)
    g.scatter_add_(1, s["y"].clamp(min=0)[:, None], g_logp[:, None])
    s["d_logits"].copy_(g * case["scale"])
    return out + [s["d_logits"]]


# ---- the library's calls ---------------------------------------------------------------------------------

def _own_scores(lib, s):
    out = [s["logp"], s["lse"], s["entropy"]]
    top = {}
    if s["case"]["op"] == "scores" and s["case"]["n_top"] > 0:
        top = {"top_logp": s["top_logp"], "top_ids": s["top_ids"]}
        out += [s["top_logp"], s["top_ids"]]
    lib.burst_lm_head_scores(s["shape"], s["logits"], y=s["y"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"], workspace=s["ws"], **top)
    return out


def _own(lib, s):
    op, out = s["case"]["op"], []
    if op in ("scores", "train"):
        out = _own_scores(lib, s)
        if op == "train":
            lib.burst_lm_head_scores_bwd(s["shape"], s["logits"], s["lse"], s["d_logits"], y=s["y"], entropy=s["entropy"], g_logp=s["g_logp"],
                                         g_lse=s["g_lse"], g_entropy=s["g_entropy"])
            out.append(s["d_logits"])
        return out
    if op == "step":
        lib.burst_attn_cache_append(s["shape"], s["cache"], s["k"], s["v"], new_rows=s["tokens"])
    if op in ("tree", "step"):
        lib.burst_attn_tree(s["shape"], s["cache"], s["tree"], s["q"], s["o"], s["lse"], s["ws"])
        out += [s["o"], s["lse"]]
    if op == "copy":
        lib.burst_attn_cache_copy_pages(s["layers"], s["moves"])
    if op in ("keep", "step"):
        lib.burst_attn_cache_keep_rows(s["layers"], s["from"], s["kept"], new_rows=s["tokens"])
    return out if op == "tree" else out + [s["K"], s["V"]]


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2509_19836_amd import binding as lib
        return _own(lib, state)
    if op == "step":
        _plain_append(state)
        return _plain_tree(state) + _plain_keep(state)
    return {"tree": _plain_tree, "copy": _plain_copy, "keep": _plain_keep, "scores": _plain_scores, "train": _plain_train}[op](state)


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _exact_scores(case, seed):
    s, out, each = _prepare_scores(case, seed), [], max(1, (1 << 26) // case["vocab"])
    n, scale = case["tokens"], case["scale"]
    for i in range(0, n, each):
        x, y = s["logits"][i:i + each].double() * scale, s["y"][i:i + each]
        logp = torch.log_softmax(x, 1)
        p, inside = logp.exp(), y >= 0
        chosen = torch.zeros_like(x)
        chosen[inside, y[inside]] = 1.0
        entropy = torch.special.entr(p).sum(1)
        part = [torch.where(inside, torch.gather(logp, 1, y.clamp(min=0)[:, None])[:, 0], 0.0), torch.logsumexp(x, 1), entropy]
        if case["op"] == "scores" and case["n_top"] > 0:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["n_top"]]
            part += [torch.gather(logp, 1, ids), ids]
        if case["op"] == "train":
            g_logp, g_lse, g_entropy = (s[name][i:i + each].double()[:, None] for name in ("g_logp", "g_lse", "g_entropy"))
            slope = torch.special.entr(p) - p * entropy[:, None]                                # of the entropy by the logits
            part.append(scale * (g_logp * inside[:, None] * (chosen - p) + g_lse * p + g_entropy * slope))
            part[-1] = part[-1] if case["tokens"] * case["vocab"] <= 3e8 else None
        out.append(part)
    return [None if parts[0] is None else torch.cat(parts) for parts in zip(*out)]


def exact(case, seed):
    if case["op"] in ("scores", "train"):
        return _exact_scores(case, seed)
    s, R = _prepare_cache(case, seed), case["page_rows"]
    rows, new, table, group = _rows(case), _new(case), s["table"].tolist(), case["q_heads"] // case["kv_heads"]
    small = case["op"] != "tree" and s["K"].numel() <= 1.2e9      # (in 64 bits, twice)
    whole = {name: s[name].double() if small else None for name in "KV"}

    def places(b, r):
        return torch.tensor([table[b][t // R] for t in r.tolist()], device="cuda"), (r % R).cuda()

    scale_of = {name: 1.0 if s[name + "_scale"] is None else s[name + "_scale"].double()[:, None] for name in "KV"}

    def put(name, x):      # numbers as the cache holds them
        if case["cache"] == "bf16":
            return x.double()
        return (x.double() / scale_of[name]).clamp(-F8_MAX, F8_MAX).float().to(torch.float8_e4m3fn).double()

    out = []
    if case["op"] in ("tree", "step"):
        words, first = [_seen_words(p) for p in _parents(case)], _first_rows(case)
        o, lse = s["o"].double(), s["lse"].double()
        for b, n in enumerate(new):
            page, r = places(b, torch.arange(rows[b]))
            K, V = (_bytes(s, name)[0][page, r] for name in "KV")
            K, V = (x.view(torch.float8_e4m3fn).double() if case["cache"] == "f8" else x.double() for x in (K, V))
            if case["op"] == "step":
                for name, x, fresh in (("K", K, s["k"]), ("V", V, s["v"])):
                    x[rows[b] - n:] = put(name, fresh[b, :n])
                    if small:
                        whole[name][0, page[rows[b] - n:], r[rows[b] - n:]] = x[rows[b] - n:]
            K, V = K * scale_of["K"], V * scale_of["V"]
            older = rows[b] if case["elsewhere"] else rows[b] - n
            hidden = torch.zeros(n, rows[b], dtype=torch.bool)
            for i in range(n):
                hidden[i, min(case["sinks"], older):min(first[b][i], older)] = True
                for t in range(older, rows[b]):
                    hidden[i, t] = not words[b][i] >> (t - older) & 1
            hidden = hidden.cuda()
            for h in range(case["q_heads"]):
                score = (s["q"][b, :n, h].double() @ K[:, h // group].T * s["scale"]).masked_fill(hidden, -math.inf)
                lse[b, h, :n] = torch.logsumexp(score, 1)
                o[b, :n, h] = torch.nan_to_num(torch.softmax(score, 1)) @ V[:, h // group]
        out = [o, lse]
    if case["op"] == "tree":
        return out
    if not small:
        return out + [None, None]
    if case["op"] == "copy":
        for name in "KV":
            before = whole[name].clone()
            for source, to, part in s["moves"].tolist():
                whole[name][:, to, :part] = before[:, source, :part]
        return [whole["K"], whole["V"]]
    for b, path in enumerate(_kept(case)):
        page, r = places(b, rows[b] - new[b] + torch.tensor(path))
        to_page, to_r = places(b, rows[b] - new[b] + torch.arange(len(path)))
        for name in "KV":
            whole[name][:, to_page, to_r] = whole[name][:, page, r].clone()
    return out + [whole["K"], whole["V"]]


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    size = {"bf16": 2, "f32": 4, "f8": 1}
    if case["op"] in ("scores", "train"):
        n, cells = case["tokens"], case["tokens"] * case["vocab"]
        nbytes = cells * size[case["logits"]] * (2 if case["op"] == "train" else 1) + n * (8 + 12 + 12 * case["n_top"])
        return {"bytes": nbytes + (12 * n if case["op"] == "train" else 0), "flops": cells * (12 if case["op"] == "train" else 6)}
    row = 2 * case["kv_heads"] * case["head_dim"] * size[case["cache"]]          # a row's keys and values
    if case["op"] == "copy":
        part = case["page_rows"] if case["pages"] > 4 else max(1, case["rows"] % case["page_rows"])
        sources = case["pages"] if case["pages"] > 4 else 1
        return {"bytes": case["layers"] * part * row * (case["pages"] + sources) + 12 * case["pages"], "flops": 0}
    nbytes = flops = 0
    if case["op"] in ("keep", "step"):
        moved = sum(sum(i != j for i, j in enumerate(path)) for path in _kept(case))
        nbytes += case.get("layers", 1) * 2 * moved * row + 4 * sum(len(path) for path in _kept(case)) + 12 * case["batch"]
    if case["op"] == "step":
        nbytes += sum(_new(case)) * case["kv_heads"] * case["head_dim"] * 2 * (2 + size[case["cache"]])
    if case["op"] in ("tree", "step"):
        Hq, d = case["q_heads"], case["head_dim"]
        for rows, n, parents, first in zip(_rows(case), _new(case), _parents(case), _first_rows(case)):
            older = rows if case["elsewhere"] else rows - n
            sinks = min(case["sinks"], older)
            hidden = [max(0, min(f, older) - sinks) for f in first]
            nbytes += (rows - min(hidden)) * row + 4 * rows // case["page_rows"]
            pairs = sum(older - h for h in hidden)
            if not case["elsewhere"]:
                pairs += sum(w.bit_count() if hasattr(w, "bit_count") else bin(w).count("1") for w in _seen_words(parents))
            nbytes += n * Hq * (d * (2 + size[case["o"]]) + 4) + 12 * n
            flops += 4 * pairs * Hq * d
    return {"bytes": nbytes, "flops": flops}
