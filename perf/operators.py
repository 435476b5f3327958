"""Rotary positions, a paged key-value cache and the attention of one new token over it, as measurable cases.

Three operators, and the run of two of them that a layer makes for every new token.  A case is a dict of plain values:

  op "rope"    turns the query and key heads of a chunk by their positions (forward), or the gradients that the backward step
               left in fp32 back again (inverse).
  op "append"  puts new keys (turned by their positions) and values into a paged cache and turns the queries on the way.
  op "decode"  attention of one new token of every sequence over the cache: (O, Lse), as a step of the ring gives them.
  op "layer"   append, then decode, with one new token a sequence: what a layer does for the next token.

batch: sequences; rows: the longest sequence's rows in the cache (the others are shorter where "ragged" is set); new: rows that a
sequence brings (at most; where "ragged" is set some bring fewer and the batch is padded).
"""
import math
import random

import torch

own = False     # whether run() makes the library's calls or computes the plain form

MAX_BYTES = 2.1e9      # of a drawn case's pass: just under the largest listed one
F8_MAX = 448.0         # the largest e4m3 number


def _case(name, op, **kw):
    case = dict(name=name, op=op, batch=1, q_heads=32, kv_heads=32, head_dim=128, rotary_dim=128, axes=1, interleaved=False, adjacent=False,
                base=10000.0)
    if op == "rope":
        case.update(new=16384, inverse=False, x="bf16", y="bf16", shards=8)
    else:
        case.update(new=1, rows=4096, ragged=False, page_rows=64, cache="bf16", by_head=False, window=0, o="bf16")
    case.update(kw)
    return case


def listed():
    return [
        # the chunk of the smallest ring of the benchmark definition: a launch and little else
        _case("rope_tiny_1k", "rope", new=256, q_heads=2, kv_heads=2, head_dim=64, rotary_dim=64, shards=4),
        # a device's chunk of a 128K-token sequence over 8 devices
        _case("rope_128k_chunk", "rope"),
        # gradients of a video model with grouped-query attention: time, height and width, fp32 in, bf16 for the projections' backward
        _case("rope_video_grads", "rope", new=32768, q_heads=64, kv_heads=8, axes=3, inverse=True, x="f32", base=500000.0),
        # the next token of a few chats
        _case("append_token_b8", "append", batch=8, kv_heads=8, rows=3001, ragged=True, page_rows=16),
        # prompts of different lengths in one padded batch, behind what their sequences hold already
        _case("append_prompts_ragged", "append", batch=4, new=4001, rows=6007, ragged=True),
        # a long video prompt into a cache of 8 bits, positions on three axes that take turns
        _case("append_video_f8", "append", q_heads=64, kv_heads=8, new=16384, rows=16384, axes=3, interleaved=True, adjacent=True,
              cache="f8", by_head=True, base=500000.0),
        # one user of a small model with 64-wide heads, a length that fits no tile and no page
        _case("decode_one_short", "decode", q_heads=12, kv_heads=12, head_dim=64, rotary_dim=64, rows=777, page_rows=16),
        # many chats of all lengths, pages of 16 rows
        _case("decode_chats_b64", "decode", batch=64, kv_heads=8, rows=4096, ragged=True, page_rows=16),
        # one device's share of a 256K-token sequence over 8 devices, joined with the others' by their Lse
        _case("decode_gqa_256k_share", "decode", q_heads=64, kv_heads=8, rows=32768, o="f32"),
        # one device's share of a 1M-token sequence over 8 devices, a key head for every query head
        _case("decode_1m_share", "decode", rows=131072, page_rows=256, by_head=True, o="f32"),
        # long contexts of many users in a cache of 8 bits
        _case("decode_f8_b32", "decode", batch=32, q_heads=64, kv_heads=8, rows=32768, ragged=True, cache="f8"),
        # a layer's work for the next token, with a sliding window
        _case("layer_b16_window", "layer", batch=16, q_heads=32, kv_heads=8, rows=16384, ragged=True, window=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["rope", "append", "decode", "decode", "layer"])
        kv = rng.choice([1, 2, 4, 5, 8, 12, 16, 32])
        group = rng.choice([g for g in (1, 1, 2, 3, 4, 7, 8, 16, 32) if kv * g <= 64])
        d = rng.choice([64, 128, 128])
        kw = dict(batch=rng.choice([1, 1, 2, 3, 7, 8, 16, 32, 64, 128]), q_heads=kv * group, kv_heads=kv, head_dim=d,
                  rotary_dim=rng.choice([d, d, d // 2, d - 16]), axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.5,
                  adjacent=rng.random() < 0.3, base=rng.choice([10000.0, 500000.0]))
        if op == "rope":
            kw["batch"] = rng.choice([1, 1, 2, 4])
            kw.update(new=_log_int(rng, 1, 131072), inverse=rng.random() < 0.5, x=rng.choice(["bf16", "f32"]),
                      y=rng.choice(["bf16", "f32"]), shards=rng.choice([1, 2, 4, 8]))
        else:
            kw.update(rows=_log_int(rng, 1, 262144), ragged=kw["batch"] > 1 and rng.random() < 0.7,
                      page_rows=rng.choice([1, 16, 16, 32, 48, 64, 128, 256]), cache=rng.choice(["bf16", "bf16", "f8"]),
                      by_head=rng.random() < 0.4, o=rng.choice(["bf16", "f32"]))
            if op == "append":
                kw["new"] = min(kw["rows"], _log_int(rng, 1, 32768))
            elif rng.random() < 0.25:
                kw["window"] = _log_int(rng, 1, kw["rows"])
        case = _case("", op, **kw)
        del case["name"]
        # what a pass moves, and the plain form's copies of the cache in 32 bits, padded to the longest sequence
        cells = 0 if op == "rope" else case["batch"] * case["rows"] * case["kv_heads"] * case["head_dim"]
        if work(case)["bytes"] <= MAX_BYTES and cells <= 1.1e9:
            return case


# ---- what a case says about its sequences ----------------------------------------------------------------

def _spread(case, most, least, salt):
    """Lengths of the case's sequences: the longest first, the others spread over the logarithm of the range."""
    if not case["ragged"]:
        return [most] * case["batch"]
    rng = random.Random(salt * 1000003 + most * 131 + case["batch"])
    return [most] + [max(least, min(most, _log_int(rng, max(least, most // 20), most))) for _ in range(case["batch"] - 1)]


def _new(case):
    return _spread(case, case["new"], 1, 1) if case["op"] == "append" else [1] * case["batch"]


def _rows(case):
    """Rows in the cache, the new ones among them."""
    return [max(n, r) for n, r in zip(_new(case), _spread(case, case["rows"], 1, 2))]


def _first(case):
    return [max(0, r - case["window"]) if case["window"] else 0 for r in _rows(case)]


def _pairs_of_axes(case):
    """The axis of each rotated pair: a quarter of them time, the rest height and width, in runs or in turns."""
    pairs = case["rotary_dim"] // 2
    if case["axes"] == 1:
        return [0] * pairs
    if case["interleaved"]:
        return [i % case["axes"] for i in range(pairs)]
    first = pairs // 4
    return [0 if i < first else 1 + (i - first) * (case["axes"] - 1) // (pairs - first) for i in range(pairs)]


# ---- inputs ----------------------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inv_freq(case):
    i = torch.arange(case["rotary_dim"] // 2, dtype=torch.float64, device="cuda")
    return (case["base"] ** (-2.0 * i / case["rotary_dim"])).float()


def _positions(case, at, gen):
    """[axes, batch, new] int32 from the tokens' places `at` [batch, new]: the place itself, or frame, line and column of a video."""
    if case["axes"] == 1:
        return at[None].to(torch.int32).contiguous()
    width, height = 40 + int(torch.randint(0, 24, (1,), generator=gen, device="cuda")), 30
    t, y, x = at // (width * height), at // width % height, at % width
    return torch.stack([t, y, x][:case["axes"]]).to(torch.int32).contiguous()


def _prepare_rope(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, n, d = case["batch"], case["new"], case["head_dim"]
    # the zigzag split's device 1: a piece near the front and one near the back of the sequence
    P, N = (n + 1) // 2, ((n + 1) // 2) * 2 * case["shards"]
    row = torch.arange(n, device="cuda")
    at = torch.where(row < P, row + (P if case["shards"] > 1 else 0), N - (2 * P if case["shards"] > 1 else P) + row - P)
    s = {"case": case, "inv_freq": _inv_freq(case), "pos": _positions(case, at[None].expand(B, n), gen)}
    for name, heads in (("q", case["q_heads"]), ("k", case["kv_heads"])):
        s[name] = torch.randn(B, n, heads, d, generator=gen, device="cuda").to(_TYPES[case["x"]])
        s[name + "_out"] = torch.empty(B, n, heads, d, device="cuda", dtype=_TYPES[case["y"]])
    return s


def _prepare_cache(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, n, Hq, Hkv, d, R = case["batch"], case["new"], case["q_heads"], case["kv_heads"], case["head_dim"], case["page_rows"]
    rows, new = _rows(case), _new(case)
    pages = [-(-r // R) for r in rows]
    cols = max(pages) + 1                                            # room for what comes
    n_pages = sum(pages) + 1
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32).tolist()
    table, at = [], 0
    for p in pages:
        table.append(order[at:at + p] + [0] * (cols - p))
        at += p
    s = {"case": case, "inv_freq": _inv_freq(case), "table": torch.tensor(table, dtype=torch.int32, device="cuda"),
         "rows": torch.tensor(rows, dtype=torch.int32, device="cuda"), "new": torch.tensor(new, dtype=torch.int32, device="cuda"),
         "first": torch.tensor(_first(case), dtype=torch.int32, device="cuda"), "max_rows": max(rows), "scale": d ** -0.5}
    f8 = case["cache"] == "f8"
    shape = (n_pages, Hkv, R, d) if case["by_head"] else (n_pages, R, Hkv, d)
    for name in ("K", "V"):
        x = torch.empty(shape, device="cuda", dtype=torch.float8_e4m3fn if f8 else torch.bfloat16)
        for i in range(0, n_pages, 4096 // R + 1):                   # keys and values of unit size, in 8 bits over a scale of their head
            part = torch.randn(x[i:i + 4096 // R + 1].shape, generator=gen, device="cuda")
            x[i:i + 4096 // R + 1] = (part * 96.0).clamp(-F8_MAX, F8_MAX).to(x.dtype) if f8 else part.to(x.dtype)
        s[name] = x.transpose(1, 2) if case["by_head"] else x        # [pages, rows, heads, head_dim]
        s[name + "_scale"] = (0.75 + 0.5 * torch.rand(Hkv, generator=gen, device="cuda")) / 96.0 if f8 else None
    s["q"] = torch.randn(B, n, Hq, d, generator=gen, device="cuda").to(torch.bfloat16)
    if case["op"] != "decode":
        s["k"], s["v"] = (torch.randn(B, n, Hkv, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        s["q_out"] = torch.zeros(B, n, Hq, d, device="cuda", dtype=torch.bfloat16)     # padding stays as it is
        s["pos"] = _positions(case, (s["rows"] - s["new"])[:, None] + torch.arange(n, device="cuda")[None], gen)
    if case["op"] != "append":
        s["o"] = torch.empty(B, 1, Hq, d, device="cuda", dtype=_TYPES[case["o"]])
        s["lse"] = torch.empty(B, Hq, 1, device="cuda")
    return s


def _descriptors(s):
    """What a user of the library fills in once, for a layer and its buffers, and keeps: sizes, the rotation, the cache, a workspace."""
    from paper_2509_19836_amd import binding as lib
    case = s["case"]
    sizes = [case[name] for name in ("batch", "q_heads", "kv_heads", "head_dim")]
    if case["op"] != "decode":
        s["shape"] = lib.shape(*sizes, case["new"], 0, 1.0)
        s["rope"] = lib.rope(s["pos"], s["inv_freq"], adjacent=case["adjacent"],
                             axis_of_pair=None if case["axes"] == 1 else _pairs_of_axes(case))
    if case["op"] != "rope":
        s["cache"] = lib.paged_cache(s["K"], s["V"], s["table"], s["rows"], k_scale=s["K_scale"], v_scale=s["V_scale"])
    if case["op"] in ("decode", "layer"):
        s["decode_shape"] = lib.shape(*sizes, 1, s["max_rows"], s["scale"])
        s["ws"] = torch.empty(lib.burst_attn_decode_workspace_bytes(s["decode_shape"]), device="cuda", dtype=torch.uint8)


def prepare(case, seed):
    s = (_prepare_rope if case["op"] == "rope" else _prepare_cache)(case, seed)
    if own:
        _descriptors(s)
    return s


# ---- the plain form --------------------------------------------------------------------------------------

def _turned(case, x, pos, inv_freq, inverse):
    """x [batch, rows, heads, head_dim] turned by its positions, in 32 bits; angles in 64 (far positions times a frequency)."""
    axis = torch.tensor(_pairs_of_axes(case), device="cuda")
    angle = pos[axis].double().permute(1, 2, 0) * inv_freq.double()                  # [batch, rows, pairs]
    c, s = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if inverse:
        s = -s
    x, R = x.float(), case["rotary_dim"]
    if case["adjacent"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([y, x[..., R:]], dim=-1)


def _plain_rope(s):
    case = s["case"]
    for name in "qk":
        s[name + "_out"].copy_(_turned(case, s[name], s["pos"], s["inv_freq"], case["inverse"]))
    return [s["q_out"], s["k_out"]]


def _plain_append(s):
    case = s["case"]
    i = torch.arange(case["new"], device="cuda")
    valid = i[None] < s["new"][:, None]
    # padding puts the sequence's last row once more
    i = torch.minimum(i[None].expand(case["batch"], -1), (s["new"] - 1)[:, None].long())
    row = (s["rows"] - s["new"]).long()[:, None] + i
    page, r = torch.gather(s["table"].long(), 1, row // case["page_rows"]), row % case["page_rows"]
    k, v = _turned(case, s["k"], s["pos"], s["inv_freq"], False), s["v"].float()
    for name, x in (("K", k), ("V", v)):
        x = torch.gather(x, 1, i[:, :, None, None].expand_as(x))
        cache = s[name]
        if case["cache"] == "f8":
            x = (x / s[name + "_scale"][:, None]).clamp(-F8_MAX, F8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
            cache = cache.view(torch.uint8)
        cache[page, r] = x.to(cache.dtype)
    q = _turned(case, s["q"], s["pos"], s["inv_freq"], False).to(torch.bfloat16)
    s["q_out"].copy_(torch.where(valid[:, :, None, None], q, s["q_out"]))
    return [s["K"], s["V"], s["q_out"]]


def _gathered(s, name):
    """Keys or values of all sequences, [batch, kv_heads, rows, head_dim] in 32 bits, padded to the longest."""
    case, cols = s["case"], -(-s["max_rows"] // s["case"]["page_rows"])
    cache = s[name].view(torch.uint8) if case["cache"] == "f8" else s[name]
    x = cache[s["table"][:, :cols].long()]
    x = x.view(torch.float8_e4m3fn) if case["cache"] == "f8" else x
    x = x.flatten(1, 2)[:, :s["max_rows"]].permute(0, 2, 1, 3).float()
    return x * s[name + "_scale"][:, None, None] if case["cache"] == "f8" else x


def _plain_decode(s, q):
    case = s["case"]
    B, Hq, Hkv, d = case["batch"], case["q_heads"], case["kv_heads"], case["head_dim"]
    score = torch.matmul(q.float().view(B, Hkv, Hq // Hkv, d), _gathered(s, "K").transpose(2, 3)) * s["scale"]
    t = torch.arange(s["max_rows"], device="cuda")
    seen = (t[None] >= s["first"][:, None]) & (t[None] < s["rows"][:, None])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, _gathered(s, "V")) / torch.where(total == 0, 1.0, total)
    s["o"].copy_(o.view(B, 1, Hq, d))
    s["lse"].copy_((top + torch.log(total)).view(B, Hq, 1))
    return [s["o"], s["lse"]]


# ---- the library's calls ---------------------------------------------------------------------------------

def _own_rope(lib, s):
    lib.burst_attn_rope(s["shape"], s["rope"], s["q"], s["q_out"], s["k"], s["k_out"], inverse=s["case"]["inverse"])
    return [s["q_out"], s["k_out"]]


def _own_append(lib, s):
    lib.burst_attn_cache_append(s["shape"], s["cache"], s["k"], s["v"], new_rows=s["new"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
    return [s["K"], s["V"], s["q_out"]]


def _own_decode(lib, s, q):
    lib.burst_attn_decode(s["decode_shape"], s["cache"], q, s["o"], s["lse"], s["ws"],
                          first_row=s["first"] if s["case"]["window"] else None)
    return [s["o"], s["lse"]]


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2509_19836_amd import binding as lib
        if op == "rope":
            return _own_rope(lib, state)
        out = [] if op == "decode" else _own_append(lib, state)
        return out if op == "append" else out + _own_decode(lib, state, state["q"] if op == "decode" else state["q_out"])
    if op == "rope":
        return _plain_rope(state)
    out = [] if op == "decode" else _plain_append(state)
    return out if op == "append" else out + _plain_decode(state, state["q"] if op == "decode" else state["q_out"])


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _exact_turned(case, x, pos, inv_freq, sign):
    """Every pair as a complex number times exp(i * sign * angle)."""
    R = case["rotary_dim"]
    y = x.double().clone()
    one = [slice(0, R, 2), slice(1, R, 2)] if case["adjacent"] else [slice(0, R // 2), slice(R // 2, R)]
    angle = torch.stack([pos[a].double() * f for a, f in zip(_pairs_of_axes(case), inv_freq.double().tolist())], dim=-1)
    z = torch.complex(y[..., one[0]], y[..., one[1]]) * torch.polar(torch.ones_like(angle), sign * angle)[:, :, None]
    y[..., one[0]], y[..., one[1]] = z.real, z.imag
    return y


def exact(case, seed):
    s = _prepare_cache(case, seed) if case["op"] != "rope" else _prepare_rope(case, seed)
    if case["op"] == "rope":
        sign = -1.0 if case["inverse"] else 1.0
        if s["q"].numel() > 3e8:                # in 64 bits, with their complex copies, a few times the memory
            return None
        return [_exact_turned(case, s[name], s["pos"], s["inv_freq"], sign) for name in "qk"]
    rows, first, new, R = _rows(case), _first(case), _new(case), case["page_rows"]
    table = s["table"].tolist()

    def places(b, r0, r1):
        r = torch.arange(r0, r1)
        return torch.tensor(table[b])[r // R].cuda(), (r % R).cuda()

    def values(name, page, r):
        x = s[name].view(torch.uint8)[page, r].view(torch.float8_e4m3fn) if case["cache"] == "f8" else s[name][page, r]
        x = x.double()
        return x * s[name + "_scale"].double()[:, None] if case["cache"] == "f8" else x

    def stored(name, x):
        if case["cache"] == "bf16":
            return x.to(torch.bfloat16).double()
        scale = s[name + "_scale"].double()[:, None]
        return (x / scale).clamp(-F8_MAX, F8_MAX).float().to(torch.float8_e4m3fn).double() * scale

    out, q, fresh = [], s["q"].double(), None
    if case["op"] != "decode":
        fresh = {"K": _exact_turned(case, s["k"], s["pos"], s["inv_freq"], 1.0), "V": s["v"].double()}
        q = torch.zeros_like(q)
        turned = _exact_turned(case, s["q"], s["pos"], s["inv_freq"], 1.0)
        whole = {name: s[name].double() if s[name].numel() <= 3e8 else None for name in "KV"}
        for b, n in enumerate(new):
            q[b, :n] = turned[b, :n]
            page, r = places(b, rows[b] - n, rows[b])
            for name in "KV":
                if whole[name] is not None:     # what the cache holds: numbers over their scale
                    whole[name][page, r] = fresh[name][b, :n] / (s[name + "_scale"].double()[:, None] if case["cache"] == "f8" else 1.0)
        out = [whole["K"], whole["V"], q]
    if case["op"] == "append":
        return out
    if fresh is not None:
        q = q.to(torch.bfloat16).double()
    o, lse = [], []
    for b in range(case["batch"]):
        page, r = places(b, first[b], rows[b])
        K, V = values("K", page, r), values("V", page, r)
        if fresh is not None:                   # the attention reads what the append left: numbers of the cache's type, queries in bf16
            for name, x in (("K", K), ("V", V)):
                x[-1] = stored(name, fresh[name][b, 0])
        group = case["q_heads"] // case["kv_heads"]
        heads_o, heads_lse = [], []
        for h in range(case["kv_heads"]):
            score = (K[:, h] @ q[b, 0, h * group:(h + 1) * group].T) * s["scale"]
            heads_lse.append(torch.logsumexp(score, 0))
            heads_o.append(torch.softmax(score, 0).T @ V[:, h])
        o.append(torch.cat(heads_o)[None])
        lse.append(torch.cat(heads_lse)[:, None])
    return out + [torch.stack(o), torch.stack(lse)]


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    Hq, Hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    size = {"bf16": 2, "f32": 4, "f8": 1}
    if case["op"] == "rope":
        tokens = case["batch"] * case["new"]
        cells = tokens * (Hq + Hkv) * d
        return {"bytes": cells * (size[case["x"]] + size[case["y"]]) + 4 * case["axes"] * tokens, "flops": 3 * cells}
    nbytes = flops = 0
    if case["op"] != "decode":
        tokens = sum(_new(case))
        nbytes += tokens * d * (2 * Hkv * (2 + size[case["cache"]]) + Hq * 4) + 4 * case["axes"] * tokens
        flops += 3 * tokens * (Hq + Hkv) * d
    if case["op"] != "append":
        seen = sum(r - f for r, f in zip(_rows(case), _first(case)))
        nbytes += 2 * seen * Hkv * d * size[case["cache"]] + 4 * seen // case["page_rows"]
        nbytes += case["batch"] * Hq * (d * (2 + size[case["o"]]) + 4)
        flops += 4 * seen * Hq * d
    return {"bytes": nbytes, "flops": flops}
