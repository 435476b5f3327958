"""decode.Draft on the CPU: what it refuses leaves the cache as it was, and what it makes of a draft's parents."""
import pytest

from tests.test_cache_binding_host import calls as recorded  # noqa: F401  (a fixture)


def cache_on_host(lib, n_pages=6, page_rows=16, batch=2, max_rows=64, lengths=(20, 3)):
    """A decode.PagedCache of tensors on the CPU."""
    import torch
    from paper_2509_19836_amd import decode
    cache = decode.PagedCache.__new__(decode.PagedCache)
    pages = torch.zeros(n_pages, page_rows, 2, 64, dtype=torch.bfloat16)
    cache.page_rows, cache.max_rows = page_rows, max_rows
    cache.table, cache.rows = torch.full((batch, -(-max_rows // page_rows)), -1, dtype=torch.int32), torch.zeros(batch, dtype=torch.int32)
    cache.lengths, cache.pages, cache.free, cache.holders = [0] * batch, [[] for _ in range(batch)], list(range(n_pages - 1, -1, -1)), [0] * n_pages
    cache.handle = lib.paged_cache(pages, torch.zeros_like(pages), cache.table, cache.rows)
    cache.layers = lib.cache_layers([cache.handle])
    cache.grow(list(lengths))
    return cache


def state(cache):
    return cache.lengths, cache.pages, cache.free, cache.holders, cache.table.tolist(), cache.rows.tolist()


@pytest.mark.parametrize("sink_rows", [-1, 1 << 31, (1 << 32) + 5])
def test_first_rows_out_of_range_are_refused(lib, recorded, sink_rows):   # noqa: F811
    """Before the draft's rows count."""
    import copy
    from paper_2509_19836_amd import decode
    cache = cache_on_host(lib)
    before = copy.deepcopy(state(cache))
    with pytest.raises(ValueError, match="sink_rows"):
        lib.tree(sink_rows=sink_rows)
    with pytest.raises(ValueError, match="sink_rows"):
        decode.Draft(cache, [[-1, 0], [-1]], window=4, sink_rows=sink_rows)
    assert state(cache) == before


def test_a_refused_draft_changes_nothing(lib, recorded):   # noqa: F811
    import copy
    from paper_2509_19836_amd import decode
    cache = cache_on_host(lib)
    before = copy.deepcopy(state(cache))
    for call, error in ((lambda: decode.Draft(cache, [[-1] * 50, [-1]]), ValueError), (lambda: decode.Draft(cache, [[-1, 0], [-1]], window=0), ValueError),
                        (lambda: decode.Draft(cache, [[-1, 0], [-1]], window=4, after=[20, 3]), ValueError), (lambda: decode.Draft(cache, [[-1, 0], [-1]], after=[20]), ValueError),
                        (lambda: decode.Draft(cache_on_host(lib, n_pages=3), [[-1] * 44, [-1]]), RuntimeError)):
        with pytest.raises(error):
            call()
    assert state(cache) == before
    short = cache_on_host(lib, n_pages=3)
    before = copy.deepcopy(state(short))
    with pytest.raises(RuntimeError, match="pages"):
        decode.Draft(short, [[-1] * 44, [-1]])
    assert state(short) == before


def test_a_draft_with_a_window(lib, recorded):   # noqa: F811
    """Words, positions, first rows and counts; the cache has grown by the draft."""
    from paper_2509_19836_amd import decode
    cache = cache_on_host(lib)
    draft = decode.Draft(cache, [[-1, 0, 1, 1, 0], [-1]], window=2, sink_rows=1)
    assert cache.lengths == [25, 4] and cache.rows.tolist() == [25, 4] and draft.counts == [5, 1]
    seen, first, tokens = draft.tree._tensors
    assert seen.tolist() == [[0b1, 0b11, 0b110, 0b1010, 0b10001], [1, 0, 0, 0, 0]]
    assert draft.positions.tolist() == [[[20, 21, 22, 22, 21], [3] * 5]] and first.tolist() == [[19, 20, 21, 21, 20], [2] * 5] and tokens.tolist() == [5, 1]
    assert draft.tree.sink_rows == 1 and draft.elsewhere.elsewhere == 1
