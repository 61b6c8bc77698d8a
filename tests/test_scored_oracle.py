"""The oracle's other scores, masks and joins against what they are in special cases."""
import numpy as np
import pytest

from oracle import attn_oracle as O


def batch(hit, app, seed=0, heads=(4, 2), dim=8, bs=4):
    g = np.random.default_rng(seed)
    need = [(h + a + bs - 1) // bs for h, a in zip(hit, app)]
    at = np.cumsum([0] + need)
    order = g.permutation(int(at[-1]))
    tables = [order[a:b] for a, b in zip(at, at[1:])]
    pool = lambda: g.standard_normal((int(at[-1]), bs, heads[1], dim))  # noqa: E731
    return hit, app, tables, bs, g.standard_normal((sum(app), heads[0], dim)), pool(), pool(), 0.4


def test_a_large_cap_and_slopes_of_zero_are_none():
    b = batch([5, 0], [3, 6])
    want = O.attend(*b)
    for kw in (dict(cap=1e9), dict(slopes=np.zeros(4)), dict(prefix=[0, 0]), dict(documents=[[], [0]])):
        for x, y in zip(O.attend(*b, **kw), want):
            np.testing.assert_allclose(x, y, rtol=1e-12, atol=1e-12)


def test_a_small_cap_makes_weights_alike():
    """Scores are then within 1e-6 of 0: lse is the logarithm of the number of keys, outputs are means of values."""
    b = batch([5], [3])
    out, lse, _, _ = O.attend(*b, cap=1e-6)
    np.testing.assert_allclose(lse, np.log(np.arange(6, 9))[:, None] * np.ones(4), atol=2e-6)
    v = b[6][np.asarray(b[2][0])].reshape(-1, 2, 8)
    np.testing.assert_allclose(out[2, 3], v[:8, 1].mean(0), atol=2e-5)


def test_two_keys_by_hand():
    """One head, two keys: the weights' ratio is the exponential of the scores' difference."""
    q, k = np.array([2.0]), [0.5, -1.5]
    pool = np.array(k).reshape(1, 2, 1, 1)
    values = np.array([1.0, 0.0]).reshape(1, 2, 1, 1)
    out, lse, _, _ = O.attend([1], [1], [[0]], 2, q.reshape(1, 1, 1), pool, values, 1.5, cap=2.0, slopes=[0.25])
    s = [2 * np.tanh(1.5 * 2 * 0.5 / 2) - 0.25, 2 * np.tanh(1.5 * 2 * -1.5 / 2)]
    np.testing.assert_allclose(out.ravel(), 1 / (1 + np.exp(s[1] - s[0])), rtol=1e-14)
    np.testing.assert_allclose(lse.ravel(), np.log(np.exp(s[0]) + np.exp(s[1])), rtol=1e-14)


def test_documents_are_requests_of_their_own():
    hit, app, tables, bs, q, k, v, scale = batch([0], [10])
    out, lse, _, _ = O.attend(hit, app, tables, bs, q, k, v, scale, documents=[[0, 4, 8]])
    for a, b in ((0, 4), (4, 8), (8, 10)):          # (documents that are whole blocks)
        part = O.attend([0], [b - a], [tables[0][a // bs:]], bs, q[a:b], k, v, scale)
        np.testing.assert_array_equal(out[a:b], part[0])
        np.testing.assert_array_equal(lse[a:b], part[1])


def test_a_prefix_of_all_tokens_is_seen_by_all():
    hit, app, tables, bs, q, k, v, scale = batch([0], [7])
    out, _, _, _ = O.attend(hit, app, tables, bs, q, k, v, scale, prefix=[7])
    keys = lambda x: x[np.asarray(tables[0])].reshape(-1, 2, 8)[:7]  # noqa: E731
    for i in range(7):
        for h in range(4):
            e = np.exp(scale * keys(k)[:, h // 2] @ q[i, h])
            np.testing.assert_allclose(out[i, h], (e / e.sum()) @ keys(v)[:, h // 2], rtol=1e-12)


@pytest.mark.parametrize("kw", [dict(), dict(cap=1.5, slopes=np.array([0, 0.1, 0.5, -0.2])), dict(prefix=[6, 2], documents=[[3, 7], [0, 1, 5]], window=4, sinks=1)])
def test_parts_joined_are_all_keys(kw):
    b = batch([6, 0], [4, 5], seed=3)
    parts = [O.attend(*b, keys=keys, **kw) for keys in ("hit", "append")]
    out, lse = O.join([x[0] for x in parts], [x[1] for x in parts])
    want = O.attend(*b, **kw)
    np.testing.assert_allclose(out, want[0], rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(lse, want[1], rtol=1e-12)


@pytest.mark.parametrize("seed", range(6))
def test_what_is_seen_from_its_definition(seed):
    g = np.random.default_rng(seed)
    window, sinks, prefix = int(g.integers(0, 6)), int(g.integers(0, 4)), int(g.integers(0, 9))
    starts = sorted(set(g.integers(0, 14, size=3).tolist()))
    document = lambda t: max([s for s in starts if s <= t], default=-1)  # noqa: E731
    for p in range(14):
        for t in range(14):
            want = t < prefix or (t <= p and (t < sinks or ((window == 0 or p - t < window) and document(t) == document(p))))
            assert O.sees(p, t, window, sinks, prefix, starts) == want
