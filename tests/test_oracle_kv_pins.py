"""Pins of oracle/kv_ref.py that do not re-type its formulas: finite differences, complex numbers, invariances, the
attention oracle."""
import numpy as np
import pytest

from oracle import attn_ref
from oracle import kv_ref as orc


def _table(npos, rot, base=10000.0):
    ang = np.arange(npos)[:, None] * base ** (-2.0 * np.arange(rot // 2) / rot)
    return np.stack((np.cos(ang), np.sin(ang)), -1)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    rng, rot, d = np.random.default_rng(1), 32, 64
    y, pos = rng.standard_normal((3, 2, d)), [0, 5, 9]
    z = orc.rotate(y, _table(10, rot), pos, rot, interleaved)
    assert np.array_equal(z[..., rot:], y[..., rot:]) and np.allclose(z[0], y[0])
    i, j = zip(*orc.pairs_of(rot, interleaved))
    ang = np.array(pos)[:, None, None] * 10000.0 ** (-2.0 * np.arange(rot // 2) / rot)
    want = (y[..., list(i)] + 1j * y[..., list(j)]) * np.exp(1j * ang)
    assert np.allclose(z[..., list(i)] + 1j * z[..., list(j)], want)
    # its transpose undoes it, and a product of two rotated rows depends on the distance alone
    assert np.allclose(orc.rotate(z, _table(10, rot), pos, rot, interleaved, -1.0), y)
    q, k = rng.standard_normal((2, 1, 1, d))
    at = lambda p, x: orc.rotate(x, _table(40, rot), [p], rot, interleaved)[0, 0]
    assert np.isclose(at(7, q) @ at(3, k), at(34, q) @ at(30, k))


@pytest.mark.parametrize("norm", [False, True])
def test_gradients_are_the_differences_of_the_forward(norm):
    rng = np.random.default_rng(2)
    T, Hq, Hkv, d, rot = 3, 4, 2, 16, 8
    x, pos, table = rng.standard_normal((T, Hq + 2 * Hkv, d)), [4, 0, 11], _table(12, rot)
    w = [1 + 0.3 * rng.standard_normal(d) if norm else None for _ in range(2)]
    g = [rng.standard_normal((T, h, d)) for h in (Hq, Hkv, Hkv)]
    loss = lambda x, wq, wk: sum((a * b).sum() for a, b in zip(g, orc.rope_qkv(x, Hq, Hkv, wq, wk, 1e-3, table, pos, rot, False)))
    dx, dwq, dwk = orc.rope_qkv_bwd(*g, x, Hq, Hkv, *w, 1e-3, table, pos, rot, False)
    eps = 1e-5
    for _ in range(5):
        u = rng.standard_normal(x.shape)
        assert np.isclose((loss(x + eps * u, *w) - loss(x - eps * u, *w)) / (2 * eps), (dx * u).sum(), rtol=1e-7, atol=1e-7)
        if norm:
            u = rng.standard_normal(d)
            assert np.isclose((loss(x, w[0] + eps * u, w[1]) - loss(x, w[0] - eps * u, w[1])) / (2 * eps), dwq @ u, rtol=1e-7, atol=1e-7)
            assert np.isclose((loss(x, w[0], w[1] + eps * u) - loss(x, w[0], w[1] - eps * u)) / (2 * eps), dwk @ u, rtol=1e-7, atol=1e-7)
    if norm:  # a row scaled by a factor gives the same output, so its gradient is orthogonal to it (eps aside)
        dx0, _, _ = orc.rope_qkv_bwd(*g, x, Hq, Hkv, *w, 0.0, table, pos, rot, False)
        assert np.allclose((dx0 * x).sum(-1)[:, :Hq + Hkv], 0.0)


def test_decode_is_the_last_row_of_causal_attention():
    rng = np.random.default_rng(3)
    Hq, Hkv, n, d, page = 4, 2, 37, 16, 8
    q, k, v = rng.standard_normal((1, Hq, n, d)), rng.standard_normal((1, Hkv, n, d)), rng.standard_normal((1, Hkv, n, d))
    want, want_lse = attn_ref.attn_ref(q, k, v, True, 0.25)
    pages = list(rng.permutation(9)[:5])
    cache = [rng.standard_normal((9, Hkv, page, d)) for _ in range(2)]
    for c, x in zip(cache, (k, v)):
        for j in range(n):
            c[pages[j // page], :, j % page] = x[0, :, j]
    o, lse = orc.decode(q[0, :, -1], *(orc.gather(c, pages, n, page) for c in cache), 0.25)
    assert np.allclose(o, want[0, :, -1]) and np.allclose(lse, want_lse[0, :, -1])
    # nothing visible, and hidden pages
    o, lse = orc.decode(q[0, :, -1], *(orc.gather(c, pages, 0, page) for c in cache), 0.25)
    assert not o.any() and np.isneginf(lse).all()
    assert orc.gather(cache[0], [-1, pages[0], 9], 24, page).shape[1] == page
