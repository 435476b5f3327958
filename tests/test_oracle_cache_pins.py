"""Pins of the fp64 reference of the rotation, the paged cache and the attention of one token: hand-worked cases, properties that the
definitions imply, differences, and the attention oracle of the ring (CPU only)."""
import numpy as np
import pytest

from oracle import burst_oracle as oc
from oracle import cache_oracle as co

FREQ = np.array([1.0, 0.25, 0.01, 0.002, 0.5, 0.125, 0.75, 0.0625], np.float32)


def _x(seed, *shape):
    return np.random.Generator(np.random.PCG64(seed)).standard_normal(shape)


def test_quarter_turn_by_hand():
    # frequency pi / 2 rounded to fp32: position 1 is a quarter turn, position 2 half a turn, up to that rounding
    f = np.array([np.pi / 2], np.float32)
    x = np.array([3.0, 5.0]).reshape(1, 1, 1, 2)
    for adjacent in (False, True):
        assert np.allclose(co.rope(x, np.array([[[1]]]), f, [0], adjacent), np.array([-5.0, 3.0]), atol=1e-6)
        assert np.allclose(co.rope(x, np.array([[[2]]]), f, [0], adjacent), np.array([-3.0, -5.0]), atol=1e-6)
        assert np.allclose(co.rope(x, np.array([[[1]]]), f, [0], adjacent, inverse=True), np.array([5.0, -3.0]), atol=1e-6)
        assert np.array_equal(co.rope(x, np.array([[[0]]]), f, [0], adjacent), x)


@pytest.mark.parametrize("adjacent", [False, True])
def test_scores_depend_on_the_distance_alone(adjacent):
    q, k = _x(1, 1, 1, 1, 24), _x(2, 1, 1, 1, 24)     # 8 pairs, 8 elements behind them
    score = lambda m, n: float((co.rope(q, np.array([[[m]]]), FREQ, [0] * 8, adjacent) * co.rope(k, np.array([[[n]]]), FREQ, [0] * 8, adjacent)).sum())
    assert abs(score(7, 3) - score(1004, 1000)) < 1e-9
    assert abs(score(7, 3) - score(8, 3)) > 1e-3
    y = co.rope(q, np.array([[[12345]]]), FREQ, [0] * 8, adjacent)
    assert np.array_equal(y[..., 16:], q[..., 16:])
    assert abs((y ** 2).sum() - (q ** 2).sum()) < 1e-9


def test_axes_turn_their_own_pairs():
    x, axes = _x(3, 2, 5, 3, 16), [0, 1, 2, 0, 1, 2, 0, 1]
    pos = np.random.Generator(np.random.PCG64(4)).integers(0, 50, (3, 2, 5))
    whole = co.rope(x, pos, FREQ, axes)
    for axis in range(3):
        alone = co.rope(x, pos[[axis]], FREQ, [0] * 8)
        mine = [i for i, a in enumerate(axes) if a == axis]
        for i in mine:
            assert np.array_equal(whole[..., [i, i + 8]], alone[..., [i, i + 8]])


@pytest.mark.parametrize("adjacent", [False, True])
def test_inverse_is_the_gradient(adjacent):
    x, g = _x(5, 1, 3, 2, 16), _x(6, 1, 3, 2, 16)
    pos = np.array([[[4, 90, 1 << 20]]])
    f = lambda z: float((co.rope(z, pos, FREQ, [0] * 8, adjacent) * g).sum())
    grad = co.rope(g, pos, FREQ, [0] * 8, adjacent, inverse=True)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = 1e-3
        assert abs((f(x + e) - f(x - e)) / 2e-3 - grad[i]) < 1e-8     # (f is linear)
    assert np.allclose(co.rope(co.rope(x, pos, FREQ, [0] * 8, adjacent), pos, FREQ, [0] * 8, adjacent, inverse=True), x, atol=1e-12)


def test_append_writes_the_new_rows_and_nothing_else():
    table = np.array([[2, 0, 9], [1, -1, 0]])          # page 9 and page -1 are none of the three
    cache = np.zeros((3, 4, 1, 2))
    x = 1 + np.arange(2 * 5 * 2).reshape(2, 5, 1, 2)
    out = co.append(cache, x, table, [6, 5], [5, 3])
    want = np.zeros_like(cache)
    for t, i in ((1, 0), (2, 1), (3, 2)):
        want[2, t] = x[0, i]
    want[0, 0], want[0, 1] = x[0, 3], x[0, 4]
    want[1, 2], want[1, 3] = x[1, 0], x[1, 1]          # row 4 of the second sequence would be in page -1
    assert np.array_equal(out, want)
    assert np.array_equal(co.append(cache, x, table, [2, 0], [4, 0])[2, :2], x[0, 2:4])   # rows before the first are left out


@pytest.mark.parametrize("page_rows", [1, 4, 7])
def test_decode_is_attention_over_the_gathered_rows(page_rows):
    rng = np.random.Generator(np.random.PCG64(7))
    n, Hq, Hkv, d = 23, 4, 2, 8
    k, v, q = _x(8, 1, n, Hkv, d), _x(9, 1, n, Hkv, d), _x(10, 1, 1, Hq, d)
    pages = -(-n // page_rows)
    table = rng.permutation(pages + 2)[None, :pages]
    K, V = np.full((pages + 2, page_rows, Hkv, d), np.nan), np.full((pages + 2, page_rows, Hkv, d), np.nan)
    for t in range(n):
        K[table[0, t // page_rows], t % page_rows], V[table[0, t // page_rows], t % page_rows] = k[0, t], v[0, t]
    for first in (0, 5, 22):
        O, lse, _, _ = co.decode(q[:, 0], K, V, table, [n], 0.3, first=[first])
        vis = (np.arange(n) >= first)[None]
        O_ref, lse_ref = oc.mha_attention_fwd(q, k, v, 0.3, vis)
        assert np.allclose(O, O_ref[:, 0], atol=1e-12) and np.allclose(lse, lse_ref[..., 0], atol=1e-12)
    O, lse, _, _ = co.decode(q[:, 0], K, V, table, [n], 0.3, first=[n])
    assert (O == 0).all() and (lse == -np.inf).all()
    # halves of the rows, merged, are the whole
    parts = [co.decode(q[:, 0], K, V, table, [hi], 0.3, first=[lo]) for lo, hi in ((0, 11), (11, n))]
    O_m, lse_m = oc.mha_lse_merge(parts[0][0][:, None], parts[0][1][..., None], parts[1][0][:, None], parts[1][1][..., None])
    O, lse, _, _ = co.decode(q[:, 0], K, V, table, [n], 0.3)
    assert np.allclose(O_m[:, 0], O, atol=1e-12) and np.allclose(lse_m[..., 0], lse, atol=1e-12)


def test_decode_scales_and_equal_keys():
    K = np.tile(np.array([1.0, 2.0]), (1, 6, 1, 1))
    V = np.arange(6.0).reshape(1, 6, 1, 1) * np.ones(2)
    O, lse, weight, size = co.decode(np.array([[[3.0, 1.0]]]), K, V, np.array([[0]]), [6], 0.5, k_scale=[2.0], v_scale=[10.0])
    assert np.allclose(O, 25.0) and np.allclose(lse, 5.0 + np.log(6)) and np.allclose(weight, 25.0) and np.allclose(size, 5.0)
