"""The oracles of drafted tokens' attention, of pages and rows that move, and of token scores with their gradient, pinned by hand-worked numbers, by other
definitions and by differences."""
import math

import numpy as np
import pytest

from oracle import burst_oracle as oc
from oracle import cache_oracle as co
from oracle import lm_head_oracle as lmo


def _x(seed, *shape):
    return np.random.Generator(np.random.PCG64(seed)).standard_normal(shape)


def test_what_a_token_sees_by_hand():
    """5 rows, the last 3 new: token 1 and 2 are siblings below token 0."""
    vis = co.tree_visible(3, 5, 5, seen=[0b001, 0b011, 0b101], first=[0, 1, 2], sinks=0)
    assert (vis == np.array([[1, 1, 1, 0, 0], [0, 1, 1, 1, 0], [0, 0, 1, 0, 1]], bool)).all()
    assert (co.tree_visible(3, 5, 5, first=[2, 2, 2], sinks=1) == np.array([[1, 0, 1, 0, 0], [1, 0, 1, 1, 0], [1, 0, 1, 1, 1]], bool)).all()
    assert (co.tree_visible(2, 3, 3, seen=[0, 0], elsewhere=True) == 1).all()                     # every row is older
    assert (co.tree_visible(2, 4, 3) == np.array([[1, 1, 1, 0], [1, 1, 1, 0]], bool)).all()        # row 3 is behind the bound
    assert co.tree_visible(0, 4, 4).shape == (0, 4)


@pytest.mark.parametrize("page_rows", [1, 4, 7])
def test_a_chain_is_causal_attention(page_rows):
    n, sq, Hq, Hkv, d = 23, 5, 4, 2, 8
    k, v, q = _x(8, 1, n, Hkv, d), _x(9, 1, n, Hkv, d), _x(10, 1, sq, Hq, d)
    pages = -(-n // page_rows)
    table = np.random.Generator(np.random.PCG64(7)).permutation(pages + 2)[None, :pages]
    K, V = np.full((pages + 2, page_rows, Hkv, d), np.nan), np.full((pages + 2, page_rows, Hkv, d), np.nan)
    for t in range(n):
        K[table[0, t // page_rows], t % page_rows], V[table[0, t // page_rows], t % page_rows] = k[0, t], v[0, t]
    O, lse, _, _ = co.tree(q, K, V, table, [n], [sq], 0.3)
    ref, lse_ref = oc.mha_attention_fwd(q, k, v, 0.3, oc.visibility(np.arange(n - sq, n), np.arange(n), True))
    assert np.allclose(O, ref, atol=1e-12) and np.allclose(lse, lse_ref, atol=1e-12)
    # a path through a tree is a chain of its own tokens
    words, path = [0b1, 0b11, 0b101, 0b1101, 0b10011], [0, 2, 3]
    O, lse, _, _ = co.tree(q, K, V, table, [n], [sq], 0.3, seen=[words])
    rows = list(range(n - sq)) + [n - sq + i for i in path]
    at = lambda x: x[:, rows]
    ref, lse_ref = oc.mha_attention_fwd(q[:, path], at(k), at(v), 0.3, oc.visibility(np.arange(n - sq, n - sq + 3), np.arange(n - sq + 3), True))
    assert np.allclose(O[:, path], ref, atol=1e-12) and np.allclose(lse[:, :, path], lse_ref, atol=1e-12)
    # one token is the step of a single token
    one = co.tree(q[:, :1], K, V, table, [n], [1], 0.3, first=[[4]])
    single = co.decode(q[:, 0], K, V, table, [n], 0.3, first=[4])
    for x, y in zip((one[0][:, 0], one[1][..., 0], one[2][:, 0], one[3][..., 0]), single):
        assert np.allclose(x, y, atol=1e-12)


def test_tokens_that_are_not_there_and_rows_that_are_none():
    q, K = np.ones((2, 2, 1, 2)), np.ones((2, 4, 1, 2))
    O, lse, weight, size = co.tree(q, K, 3 * K, np.array([[0], [-1]]), [4, 4], [1, 9], 0.5)
    assert np.isnan(O[0, 1]).all() and np.isnan(lse[0, 0, 1]) and np.allclose(O[0, 0], 3) and np.isclose(lse[0, 0, 0], 1 + math.log(4))
    assert (O[1] == 0).all() and (lse[1] == -np.inf).all() and np.allclose(weight[0, 0], 3) and np.isclose(size[0, 0, 0], 1)


def test_moves_by_hand():
    cache = np.arange(12).reshape(3, 4, 1)
    got = co.copy_pages(cache, [[0, 2, 3], [1, 1, 4], [0, 7, 4], [-1, 1, 4], [0, 1, -2]])
    assert got[2, :, 0].tolist() == [0, 1, 2, 11] and (got[:2] == cache[:2]).all()
    table, rows = np.array([[2, 0, -1], [1, 1, 1]]), [7, 3]
    got = co.keep_rows(cache, table, rows, [[3, 0, 4, 0, 0], [1, 0, 0, 0, 0]], [5, 2], [3, 2])
    # sequence 0: rows 2 .. 6 are 10, 11 of page 2 and 0, 1, 2 of page 0; its new rows 3, 0 and 4 to their front.  sequence 1: rows 1, 2 of page 1 change places
    assert got[2, :, 0].tolist() == [8, 9, 1, 10] and got[0, :, 0].tolist() == [2, 1, 2, 3] and got[1, :, 0].tolist() == [4, 6, 5, 7]
    got = co.keep_rows(cache, table, rows, [[5, -1, 0, 0, 0], [0, 0, 0, 0, 0]], [5, 2], [2, 0])   # places outside: as they were
    assert (got == cache).all()


def test_scores_by_hand():
    x = np.log(np.array([[1.0, 2.0, 4.0, 1.0], [3.0, 3.0, 3.0, 3.0]]))
    s = lmo.scores(x, [1, 9], 3)
    assert np.allclose(s["lse"], np.log([8, 12])) and np.allclose(s["logp"], [np.log(0.25), 0]) and np.allclose(s["entropy"], [1.75 * np.log(2), np.log(4)])
    assert s["top_ids"].tolist() == [[2, 1, 0], [0, 1, 2]] and np.allclose(s["top_logp"], np.log([[0.5, 0.25, 0.125], [0.25] * 3]))
    s = lmo.scores(x, scale=2.0)
    assert np.allclose(s["lse"], np.log([22, 36]))
    s = lmo.scores(np.array([[-np.inf, 0.0, -np.inf], [-np.inf] * 3]), [0, 1], 2)
    assert s["lse"].tolist() == [0, -np.inf] and s["entropy"].tolist() == [0, 0] and s["logp"].tolist() == [-np.inf, -np.inf]
    assert s["top_ids"].tolist() == [[1, 0], [0, 1]] and s["top_logp"].tolist() == [[0, -np.inf], [-np.inf, -np.inf]]


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_scores_gradient_by_differences_and_by_autograd(scale):
    import torch
    n, v, k = 3, 7, 2
    x, y = _x(1, n, v), np.array([2, -1, 6])
    g = {name: _x(i + 2, *size) for i, (name, size) in enumerate((("logp", (n,)), ("lse", (n,)), ("entropy", (n,)), ("top_logp", (n, k))))}
    ids = lmo.scores(x, y, k, scale)["top_ids"]

    def total(x):
        s = lmo.scores(x, y, k, scale)
        assert (s["top_ids"] == ids).all()
        return sum((g[name] * s[name]).sum() for name in g)
    grad = lmo.scores_bwd(x, y, ids, g["logp"], g["lse"], g["entropy"], g["top_logp"], scale)
    eps, num = 1e-6, np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += eps
        down[i] -= eps
        num[i] = (total(up) - total(down)) / (2 * eps)
    assert np.allclose(grad, num, atol=1e-8)
    t = torch.from_numpy(x).requires_grad_()
    logp = torch.log_softmax(scale * t, 1)
    out = (torch.from_numpy(g["lse"]) * torch.logsumexp(scale * t, 1)).sum() - (torch.from_numpy(g["entropy"]) * (logp.exp() * logp).sum(1)).sum()
    out = out + (torch.from_numpy(g["top_logp"]) * logp.gather(1, torch.from_numpy(ids))).sum()
    out = out + sum(float(g["logp"][i]) * logp[i, y[i]] for i in range(n) if y[i] >= 0)
    out.backward()
    assert np.allclose(grad, t.grad.numpy(), atol=1e-12)


def test_scores_gradient_of_masked_and_repeated_words():
    x = np.array([[0.5, -np.inf, 0.25, 1.0], [-np.inf] * 4])
    grad = lmo.scores_bwd(x, [3, 0], np.array([[3, 3], [0, 1]]), g_logp=np.array([1.0, 1.0]), g_top=np.array([[2.0, 0.5], [1.0, 1.0]]))
    p = np.exp(x[0] - np.log(np.exp(x[0]).sum()))
    assert np.allclose(grad[0], [-3.5 * p[0], 0, -3.5 * p[2], 3.5 - 3.5 * p[3]]) and (grad[1] == 0).all()
    grad = lmo.scores_bwd(x, top_ids=np.array([[0, -1], [0, 4]]), g_top=np.array([[1.0, 5.0], [1.0, 1.0]]))   # a word that is none takes its gradient with it
    assert np.allclose(grad[0], [1 - p[0], 0, -p[2], -p[3]]) and (grad[1] == 0).all()
