"""Token by token after a ring's forward pass: the pages of a device's cache, and a token's step over one device or all of a ring.

A device keeps the keys (turned by their positions) and values that it holds of each sequence in a paged cache.  Pages are handed out
here, on the host; what is computed are calls into the C ABI: burst_attn_cache_append, burst_attn_decode and, over the devices of a ring,
burst_attn_lse_merge.  The order of a sequence's rows in the cache plays no part in its attention, so a device appends what it holds
of the sequence (a zigzag or striped chunk, for instance) as it comes, with the rows' positions in the rotation.
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
        self.handle = lib.paged_cache(k, v, self.table, self.rows, k_scale, v_scale)

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
                fresh = [self.free.pop() for _ in range(n)]
                at = len(self.pages[b])
                self.table[b, at:at + n] = torch.tensor(fresh, dtype=torch.int32)
                self.pages[b] += fresh
        self.rows.copy_(torch.tensor(lengths, dtype=torch.int32))

    def release(self, b):
        """Sequence b is over: its pages are free again, on the current stream."""
        self.free += reversed(self.pages[b])
        self.pages[b], self.lengths[b] = [], 0
        self.table[b] = -1
        self.rows[b] = 0


def append(cache, q, k, v, rope, q_out, new_rows=None, stream=None):
    """The rows that the cache has grown by: k (turned) and v into it, q (turned) into q_out; new_rows: those numbers as an int32 tensor on the
    device, that lives until the call has run (None: all rows of k)."""
    B, n, Hq, d = q.shape
    lib.burst_attn_cache_append(lib.shape(B, Hq, k.shape[2], d, n, 0, 1.0), cache.handle, k, v, new_rows=new_rows, rope=rope, q=q,
                                q_out=q_out, stream=stream)


def workspace(cache, q_heads):
    """A workspace for the attention over this cache; calls that share one are ordered on one stream."""
    kv_heads, d = cache.handle._tensors[0].shape[2:]
    shp = lib.shape(len(cache.lengths), q_heads, kv_heads, d, 1, cache.max_rows, 1.0)
    return torch.empty(lib.burst_attn_decode_workspace_bytes(shp), device=cache.rows.device, dtype=torch.uint8)


def attend(cache, q, scale, o, lse, ws, first_row=None, stream=None):
    """One new token of each sequence, q [batch, 1, q_heads, head_dim] as append left it, over all rows of the cache: o, lse.  The call's bound
    of the rows is max_rows, whatever the sequences have, so that a captured one serves them as they grow; a program that knows less to be enough
    calls binding.burst_attn_decode with that, which is faster for short sequences in a large cache."""
    B, _, Hq, d = q.shape
    shp = lib.shape(B, Hq, cache.handle._tensors[0].shape[2], d, 1, cache.max_rows, scale)
    lib.burst_attn_decode(shp, cache.handle, q, o, lse, ws, first_row=first_row, stream=stream)


def ring_token(caches, owner, q, k, v, rope, scale, q_out, o_acc, lse_acc, o_part, lse_part, ws, stream=None):
    """A token of each sequence whose rows are dealt over a ring's devices, here caches on one GPU: device `owner`, whose cache has grown by
    a row, takes the new key and value; every device attends over the rows that it holds, and what they find is joined.  o_acc [batch, 1,
    q_heads, head_dim] and lse_acc [batch, q_heads, 1] must hold (0, -inf) on entry; they hold (O, Lse) over all devices on return."""
    append(caches[owner], q, k, v, rope, q_out, stream=stream)
    B, _, Hq, d = q.shape
    for cache in caches:
        attend(cache, q_out, scale, o_part, lse_part, ws, stream=stream)
        lib.burst_attn_lse_merge(lib.shape(B, Hq, k.shape[2], d, 1, 0, scale), o_acc, lse_acc, o_part, lse_part, stream=stream)
