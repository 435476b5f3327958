"""Token by token after a ring's forward pass: the pages of a device's cache, and a token's step over one device or all of a ring.

A device keeps the keys (turned by their positions) and values that it holds of each sequence in a paged cache.  Pages are handed out
here, on the host; what is computed are calls into the C ABI: burst_attn_cache_append, burst_attn_decode and, over the devices of a ring,
burst_attn_lse_merge.  The order of a sequence's rows in the cache plays no part in its attention, so a device appends what it holds
of the sequence (a zigzag or striped chunk, for instance) as it comes, with the rows' positions in the rotation.

Several tokens of a sequence at once, guesses at how it goes on that share what they begin with, are a Draft: they are appended as any rows are,
attend_tree lets each see the ones that it continues (burst_attn_tree), burst_lm_head_scores says what the model makes of them, and PagedCache.keep
leaves the accepted ones (burst_attn_cache_keep_rows).  PagedCache.fork lets sequences begin with another one's rows (burst_attn_cache_copy_pages).
"""
import torch

from . import binding as lib


class PagedCache:
    """Pages of page_rows rows for `batch` sequences of up to max_rows rows each on the current device: bf16, or float8_e4m3fn over scales
    of the key heads.  In memory a page has its rows head by head, the order that is read fastest.  The keys and values are one layer's; another
    layer's, in tensors of the same n_pages and page_rows, go by the same numbers: binding.paged_cache(k, v, cache.table, cache.rows)."""

    def __init__(self, n_pages, page_rows, batch, kv_heads, head_dim, max_rows, dtype=torch.bfloat16, k_scale=None, v_scale=None):
        device = torch.device("cuda", torch.cuda.current_device())
        self.page_rows, self.max_rows = page_rows, max_rows
        cols = max(1, -(-max_rows // page_rows))
        k, v = (torch.empty(n_pages, kv_heads, page_rows, head_dim, device=device, dtype=dtype).transpose(1, 2) for _ in range(2))
        self.table = torch.full((batch, cols), -1, device=device, dtype=torch.int32)
        self.rows = torch.zeros(batch, device=device, dtype=torch.int32)
        self.lengths = [0] * batch              # the host's copy of rows
        self.pages = [[] for _ in range(batch)]
        self.free = list(range(n_pages - 1, -1, -1))
        self.holders = [0] * n_pages            # sequences that have a page: several have full ones alone
        self.handle = lib.paged_cache(k, v, self.table, self.rows, k_scale, v_scale)
        self.layers = lib.cache_layers([self.handle])

    def _take(self, n):
        fresh = [self.free.pop() for _ in range(n)]
        for page in fresh:
            self.holders[page] = 1
        return fresh

    def _give(self, pages):
        for page in reversed(pages):
            self.holders[page] -= 1
            if self.holders[page] == 0:
                self.free.append(page)

    def grow(self, new_rows):
        """Room for new_rows[b] more rows of each sequence, which count from now on: the next append (in every layer that goes by the table) fills
        them, on the current stream, for which the host waits here.  Raises, and changes nothing, where pages run out or a sequence would
        pass max_rows."""
        lengths = [n + m for n, m in zip(self.lengths, new_rows, strict=True)]
        if min(new_rows) < 0 or max(lengths) > self.max_rows:
            raise ValueError(f"a sequence has 0 to {self.max_rows} rows")
        need = [-(-n // self.page_rows) - len(p) for n, p in zip(lengths, self.pages)]
        if sum(max(0, n) for n in need) > len(self.free):
            raise RuntimeError(f"{sum(max(0, n) for n in need)} pages asked for, {len(self.free)} are free")
        self.lengths = lengths
        for b, n in enumerate(need):
            if n > 0:
                fresh = self._take(n)
                at = len(self.pages[b])
                self.table[b, at:at + n] = torch.tensor(fresh, dtype=torch.int32)
                self.pages[b] += fresh
        self.rows.copy_(torch.tensor(lengths, dtype=torch.int32))

    def release(self, b):
        """Sequence b is over: its pages that no other has are free again, on the current stream."""
        self._give(self.pages[b])
        self.pages[b], self.lengths[b] = [], 0
        self.table[b] = -1
        self.rows[b] = 0

    def fork(self, source, targets, layers=None):
        """The empty sequences `targets` begin with the rows that `source` has, on the current stream: they share its full pages, and the rows of the last,
        partly filled one are copied into a page of each one's own, in all layers that go by the table (binding.cache_layers; None: this one alone).
        Raises, and changes nothing, where pages run out."""
        targets = list(targets)
        if len({source, *targets}) != len(targets) + 1 or min([source, *targets]) < 0 or any(self.lengths[b] for b in targets):
            raise ValueError("empty sequences expected, each of them once")
        full, over = divmod(self.lengths[source], self.page_rows)
        if over and len(targets) > len(self.free):
            raise RuntimeError(f"{len(targets)} pages asked for, {len(self.free)} are free")
        if over and targets:
            moves = [[self.pages[source][full], page, over] for page in reversed(self.free[-len(targets):])]
            lib.burst_attn_cache_copy_pages(self.layers if layers is None else layers, torch.tensor(moves, dtype=torch.int32).to(self.rows.device))
        shared = self.pages[source][:full]
        for b in targets:
            for page in shared:
                self.holders[page] += 1
            own = self._take(1) if over else []
            self.pages[b], self.lengths[b] = shared + own, self.lengths[source]
            self.table[b] = self.table[source]
            if own:
                self.table[b, full] = own[0]
            self.rows[b] = self.lengths[b]

    def keep(self, new_rows, kept, layers=None):
        """Of the last new_rows[b] rows of each sequence those stay that kept[b] names (0: the first of them), in its order, and the pages behind them are
        free again, in all layers that go by the table (binding.cache_layers; None: this one alone), on the current stream, for which the host waits here."""
        new_rows, kept = list(new_rows), [list(rows) for rows in kept]
        if len(new_rows) != len(self.lengths) or len(kept) != len(new_rows):
            raise ValueError(f"new rows and kept rows of {len(self.lengths)} sequences expected")
        for b, (n, rows) in enumerate(zip(new_rows, kept)):
            if not 0 <= n <= min(self.lengths[b], lib.BURST_TREE_MAX_TOKENS) or len(rows) > n or any(not 0 <= r < n for r in rows):
                raise ValueError(f"sequence {b}: rows {rows} of its last {n} of {self.lengths[b]}")
            if n and any(self.holders[page] > 1 for page in self.pages[b][(self.lengths[b] - n) // self.page_rows:]):
                raise ValueError(f"sequence {b} shares pages of its last {n} rows with another")
        sq = max(new_rows)
        if sq == 0:
            return
        on_device = lambda x: torch.tensor(x, dtype=torch.int32).to(self.rows.device)
        lib.burst_attn_cache_keep_rows(self.layers if layers is None else layers, on_device([rows + [-1] * (sq - len(rows)) for rows in kept]),
                                       on_device([len(rows) for rows in kept]), new_rows=on_device(new_rows))
        for b, (n, rows) in enumerate(zip(new_rows, kept)):
            self.lengths[b] += len(rows) - n
            have = -(-self.lengths[b] // self.page_rows)
            if have < len(self.pages[b]):
                self._give(self.pages[b][have:])
                del self.pages[b][have:]
                self.table[b, have:] = -1
        self.rows.copy_(torch.tensor(self.lengths, dtype=torch.int32))


class Draft:
    """Drafted tokens of every sequence, behind its rows in the cache, which has grown by them: parents[b][i] is the number of the token that token i
    of sequence b continues, a lower one, or -1: the sequence's last row.  A token sees the tokens that it continues, itself and the older rows; with a
    window, of all these the last `window` on the way to it, and the first sink_rows rows of the sequence (which are not among the drafted ones).
    counts: the tokens of each sequence; new_rows: those on the device; positions int32 [1, batch, tokens], for the rotation, from after[b] on (None: the
    rows that the sequence had; a window needs that they lie in the cache in their order); tree: binding.tree; elsewhere: that of the other devices of a ring."""

    def __init__(self, cache, parents, window=None, sink_rows=0, after=None):
        parents = [list(p) for p in parents]
        if cache.handle._device != torch.cuda.current_device():
            raise ValueError(f"the cache is on cuda:{cache.handle._device}, the current device is cuda:{torch.cuda.current_device()}")
        if len(parents) != len(cache.lengths) or any(not -1 <= up < i for p in parents for i, up in enumerate(p)):
            raise ValueError(f"for each token of {len(cache.lengths)} sequences the number of an earlier one or -1 expected")
        self.counts = [len(p) for p in parents]
        sq = max(self.counts)
        if not 0 < sq <= lib.BURST_TREE_MAX_TOKENS or (window is not None and (window < 1 or after is not None)):
            raise ValueError(f"1 to {lib.BURST_TREE_MAX_TOKENS} tokens of a sequence and a window of a row or more expected, and no window with rows elsewhere")
        self.parents, older = parents, list(cache.lengths if after is None else after)
        seen, depth = [], []
        for p in parents:
            words, deep = [], []
            for i, up in enumerate(p):
                deep.append(0 if up < 0 else deep[up] + 1)
                words.append((0 if up < 0 else words[up]) | 1 << i)
            if window is not None:
                words = [sum(1 << j for j in range(i + 1) if w >> j & 1 and deep[i] - deep[j] < window) for i, w in enumerate(words)]
            seen.append([w - (1 << 64) if w >> 63 else w for w in words] + [0] * (sq - len(p)))
            depth.append(deep + [0] * (sq - len(p)))
        places = [[n + i for i in deep] for n, deep in zip(older, depth, strict=True)]
        device = cache.rows.device
        first = None if window is None else torch.tensor([[max(0, t - window + 1) for t in row] for row in places], dtype=torch.int32).to(device)
        self.positions = torch.tensor([places], dtype=torch.int32).to(device)
        self.new_rows = torch.tensor(self.counts, dtype=torch.int32).to(device)
        self.tree = lib.tree(torch.tensor(seen, dtype=torch.int64).to(device), first, self.new_rows, sink_rows=0 if window is None else sink_rows)
        self.elsewhere = lib.tree(tokens=self.new_rows, elsewhere=True)
        cache.grow(self.counts)   # (last: a draft that is refused leaves the cache as it was)

    def agreed(self, words, likeliest):
        """The path of each sequence through its draft where every token is the likeliest word after the one before: token 0, which is given, then of the
        tokens that continue the path the one whose word (words[b][i]) is likeliest[b] of the path's last.  What keep takes; the word after the path is
        likeliest[b] of its last."""
        paths = []
        for p, has, best in zip(self.parents, words, likeliest, strict=True):
            path = [0] if p else []
            while path:
                on = [i for i, up in enumerate(p) if up == path[-1] and has[i] == best[path[-1]]]
                if not on:
                    break
                path.append(on[0])
            paths.append(path)
        return paths


def append(cache, q, k, v, rope, q_out, new_rows=None, stream=None):
    """The rows that the cache has grown by: k (turned) and v into it, q (turned) into q_out; new_rows: those numbers as an int32 tensor on the
    device, that lives until the call has run (None: all rows of k)."""
    B, n, Hq, d = q.shape
    lib.burst_attn_cache_append(lib.shape(B, Hq, k.shape[2], d, n, 0, 1.0), cache.handle, k, v, new_rows=new_rows, rope=rope, q=q,
                                q_out=q_out, stream=stream)


def workspace(cache, q_heads, tokens=0):
    """A workspace for the attention over this cache; calls that share one are ordered on one stream.  tokens: of drafts of up to so many."""
    kv_heads, d = cache.handle._tensors[0].shape[2:]
    shape = lambda sq: lib.shape(len(cache.lengths), q_heads, kv_heads, d, sq, cache.max_rows, 1.0)
    n = max(lib.burst_attn_decode_workspace_bytes(shape(1)), *(lib.burst_attn_tree_workspace_bytes(shape(sq)) for sq in range(1, tokens + 1)), 0)
    return torch.empty(n, device=cache.rows.device, dtype=torch.uint8)


def attend(cache, q, scale, o, lse, ws, first_row=None, stream=None):
    """One new token of each sequence, q [batch, 1, q_heads, head_dim] as append left it, over all rows of the cache: o, lse.  The call's bound
    of the rows is max_rows, whatever the sequences have, so that a captured one serves them as they grow; a program that knows less to be enough
    calls binding.burst_attn_decode with that, which is faster for short sequences in a large cache."""
    B, _, Hq, d = q.shape
    shp = lib.shape(B, Hq, cache.handle._tensors[0].shape[2], d, 1, cache.max_rows, scale)
    lib.burst_attn_decode(shp, cache.handle, q, o, lse, ws, first_row=first_row, stream=stream)


def attend_tree(cache, draft, q, scale, o, lse, ws, layer=None, elsewhere=False, stream=None):
    """The tokens of a draft, q [batch, tokens, q_heads, head_dim] as append left it, over the rows that each sees: o, lse.  layer: the handle of a layer
    that goes by the cache's table (None: the cache's own); elsewhere: another cache of a ring has grown by the draft.  The rows of a shorter draft's missing
    tokens are left as they were.  As in attend the call's bound of the rows is max_rows."""
    layer = cache.handle if layer is None else layer
    B, n, Hq, d = q.shape
    lib.burst_attn_tree(lib.shape(B, Hq, layer._tensors[0].shape[2], d, n, cache.max_rows, scale), layer, draft.elsewhere if elsewhere else draft.tree, q, o, lse, ws, stream=stream)


def ring_token(caches, owner, q, k, v, rope, scale, q_out, o_acc, lse_acc, o_part, lse_part, ws, stream=None):
    """A token of each sequence whose rows are dealt over a ring's devices, here caches on one GPU: device `owner`, whose cache has grown by
    a row, takes the new key and value; every device attends over the rows that it holds, and what they find is joined.  o_acc [batch, 1,
    q_heads, head_dim] and lse_acc [batch, q_heads, 1] must hold (0, -inf) on entry; they hold (O, Lse) over all devices on return."""
    append(caches[owner], q, k, v, rope, q_out, stream=stream)
    B, _, Hq, d = q.shape
    for cache in caches:
        attend(cache, q_out, scale, o_part, lse_part, ws, stream=stream)
        lib.burst_attn_lse_merge(lib.shape(B, Hq, k.shape[2], d, 1, 0, scale), o_acc, lse_acc, o_part, lse_part, stream=stream)


def ring_draft(caches, owner, draft, q, k, v, rope, scale, q_out, o_acc, lse_acc, o_part, lse_part, ws, stream=None):
    """As ring_token, for a draft by which the cache of device `owner` has grown: the buffers have its tokens where those have one.  Rows of a shorter draft's
    missing tokens are unspecified."""
    append(caches[owner], q, k, v, rope, q_out, new_rows=draft.new_rows, stream=stream)
    B, n, Hq, d = q.shape
    for i, cache in enumerate(caches):
        attend_tree(cache, draft, q_out, scale, o_part, lse_part, ws, elsewhere=i != owner, stream=stream)
        lib.burst_attn_lse_merge(lib.shape(B, Hq, k.shape[2], d, n, 0, scale), o_acc, lse_acc, o_part, lse_part, stream=stream)
