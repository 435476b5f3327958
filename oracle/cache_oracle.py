"""fp64 reference of the rotation by positions, the paged cache and the attention of one new token (test infrastructure only).

Plain numpy, written from the definitions in include/burst_attn_cache.h; shares no code with the HIP path and never imports it.
"""
import numpy as np

F8_MAX = 448.0


def pair_elements(rotary_dim, adjacent):
    """Elements (first, second) of each pair of a head."""
    i = np.arange(rotary_dim // 2)
    return (2 * i, 2 * i + 1) if adjacent else (i, i + rotary_dim // 2)


def angles(positions, inv_freq, axis_of_pair):
    """[batch, rows, pairs] from positions [axes, batch, rows]: exact products of whole numbers and fp32 frequencies."""
    pos = np.asarray(positions)[np.asarray(axis_of_pair, dtype=np.int64)]             # [pairs, batch, rows]
    return np.moveaxis(pos.astype(np.longdouble), 0, -1) * np.asarray(inv_freq, np.float32).astype(np.longdouble)


def rope(x, positions, inv_freq, axis_of_pair, adjacent=False, inverse=False):
    """x [batch, rows, heads, head_dim] turned pair by pair."""
    a = angles(positions, inv_freq, axis_of_pair)
    c, s = np.cos(a).astype(np.float64)[:, :, None], np.sin(a).astype(np.float64)[:, :, None]
    if inverse:
        s = -s
    first, second = pair_elements(2 * len(axis_of_pair), adjacent)
    y = np.array(x, np.float64)
    x1, x2 = y[..., first], y[..., second]
    y[..., first], y[..., second] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def slots(table, page_rows, b, rows):
    """(page, row of the page) of rows of sequence b, as the table says it, pages that are none included."""
    rows = np.asarray(rows, np.int64)
    return np.asarray(table)[b, rows // page_rows].astype(np.int64), rows % page_rows


def new_places(table, page_rows, n_pages, rows, new):
    """For each sequence the (index of the new row, page, row of the page) that an append writes."""
    most = np.asarray(table).shape[1] * page_rows
    for b in range(len(rows)):
        have = min(max(int(rows[b]), 0), most)
        for i in range(int(new[b])):
            t = have - int(new[b]) + i
            if t < 0:
                continue
            page, r = slots(table, page_rows, b, t)
            if 0 <= page < n_pages:
                yield b, i, int(page), int(r)


def append(cache, x, table, rows, new, scale=None):
    """cache [pages, page_rows, kv_heads, head_dim] with the new rows of x [batch, sq, kv_heads, head_dim] in it, as numbers over their
    head's scale, not yet rounded."""
    out = np.array(cache, np.float64)
    for b, i, page, r in new_places(table, out.shape[1], out.shape[0], rows, new):
        out[page, r] = x[b, i] if scale is None else np.clip(x[b, i] / np.asarray(scale, np.float64)[:, None], -F8_MAX, F8_MAX)
    return out


def decode(q, k, v, table, rows, scale, first=None, max_rows=None, k_scale=None, v_scale=None):
    """q [batch, q_heads, head_dim] over the cache k, v [pages, page_rows, kv_heads, head_dim]: O, Lse [batch, q_heads], and for tolerances
    the sum of P |V| and the largest sum of |q| |K| of each head."""
    B, Hq, d = q.shape
    n_pages, page_rows, Hkv, _ = k.shape
    group = Hq // Hkv
    ks = np.ones(Hkv) if k_scale is None else np.asarray(k_scale, np.float64)
    vs = np.ones(Hkv) if v_scale is None else np.asarray(v_scale, np.float64)
    O, lse, weight, size = np.zeros((B, Hq, d)), np.full((B, Hq), -np.inf), np.zeros((B, Hq, d)), np.zeros((B, Hq))
    for b in range(B):
        hi = min(max(int(rows[b]), 0), table.shape[1] * page_rows)
        hi = hi if max_rows is None else min(hi, max_rows)
        lo = 0 if first is None else max(int(first[b]), 0)
        if hi <= lo:
            continue
        page, r = slots(table, page_rows, b, np.arange(lo, hi))
        there = (page >= 0) & (page < n_pages)
        page, r = page[there], r[there]
        if page.size == 0:
            continue
        K, V = k[page, r].astype(np.float64) * ks[:, None], v[page, r].astype(np.float64) * vs[:, None]   # [rows, kv_heads, head_dim]
        for h in range(Hq):
            s = K[:, h // group] @ q[b, h].astype(np.float64) * scale
            top = s.max()
            if top == -np.inf:
                continue
            p = np.exp(s - top)
            lse[b, h] = top + np.log(p.sum())
            O[b, h] = p @ V[:, h // group] / p.sum()
            weight[b, h] = p @ np.abs(V[:, h // group]) / p.sum()
            size[b, h] = (np.abs(K[:, h // group]) @ np.abs(q[b, h].astype(np.float64))).max() * scale
    return O, lse, weight, size
