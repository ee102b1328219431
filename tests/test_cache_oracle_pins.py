"""Pins of the rotation and cache oracle (CPU): worked examples, properties of the definition, the attention oracle."""
import numpy as np
import pytest

import oracle
from oracle import cache


def test_a_quarter_turn():
    x = np.array([[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]])
    f = [np.pi / 2, np.pi]                                          # position 1: a quarter and a half turn
    np.testing.assert_allclose(cache.rotate(x, [1], f), [[-3, -2, 1, -4, 5, 6]], atol=1e-6)
    np.testing.assert_allclose(cache.rotate(x, [1], f, adjacent=True), [[-2, 1, -3, -4, 5, 6]], atol=1e-6)
    np.testing.assert_allclose(cache.rotate(x, [0], f), x)


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_is_orthogonal_and_scores_depend_on_distance(adjacent):
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 16))
    f = 10000.0 ** (-np.arange(6) / 6)
    for p in (0, 5, 123456):
        y = cache.rotate(q, [p], f, adjacent)
        np.testing.assert_allclose(np.linalg.norm(y), np.linalg.norm(q))
        np.testing.assert_allclose(cache.rotate(y, [p], f, adjacent, back=True), q, atol=1e-12)
    score = lambda i, j: cache.rotate(q, [i], f, adjacent)[0] @ cache.rotate(k, [j], f, adjacent)[0]
    np.testing.assert_allclose(score(7, 3), score(1007, 1003), atol=1e-11)


def test_far_positions():
    """2^31 - 1 times 1 radian, with the cosine of a known reduction."""
    n = 2 ** 31 - 1
    turns, two_pi = divmod(n * 10 ** 40, 62831853071795864769252867665590057683943)      # 2 pi in 40 digits
    y = cache.rotate(np.array([[1.0, 0.0]]), [n], [1.0])
    np.testing.assert_allclose(y, [[np.cos(two_pi / 1e40), np.sin(two_pi / 1e40)]], atol=1e-9)


@pytest.mark.parametrize("zigzag", [False, True])
def test_tokens_of_the_ranks(zigzag):
    every = cache.tokens(1024, 4, 0, 4, zigzag)
    assert sorted(every) == list(range(1024))
    for n in range(4):
        assert list(cache.tokens(1024, 4, n, n + 1, zigzag)) == list(every[n * 256:(n + 1) * 256])
    if zigzag:
        assert every[0] == 0 and every[128] == 7 * 128 and every[256] == 128


def test_cache_against_the_attention_oracle():
    rng = np.random.default_rng(1)
    B, Zkv, g, A, page, W = 2, 2, 3, 64, 5, 4
    n = [17, 9]
    K, V = rng.standard_normal((2, B, Zkv, 17, A))
    table = np.array([[7, 1, 4, 2], [0, 6, 3, 5]])
    Kc = Vc = np.full((8, Zkv, page, A), np.nan)
    _, Kc, Vc = cache.append(K, V, Kc, Vc, table, n, counts=n)
    assert np.isnan(Kc[5]).all() and np.isnan(Kc[2, :, 2:]).all() and not np.isnan(Kc[2, :, :2]).any()
    np.testing.assert_array_equal(Kc[4, :, 3], K[0, :, 13])
    Q = rng.standard_normal((B, Zkv * g, 1, A))
    O, LSE = cache.attend(Q, Kc, Vc, table, n)
    for b in range(B):
        k, v = (np.repeat(x[b:b + 1, :, :n[b]], g, axis=1) for x in (K, V))
        o, l = oracle.forward(np.ascontiguousarray(Q[b:b + 1]), np.ascontiguousarray(k), np.ascontiguousarray(v))[:2]
        np.testing.assert_allclose(O[b:b + 1], o, atol=1e-12)
        np.testing.assert_allclose(LSE[b:b + 1], l, atol=1e-12)


def test_pages_that_are_not_held_and_empty_sequences():
    rng = np.random.default_rng(2)
    Kc, Vc = rng.standard_normal((2, 4, 1, 2, 64))
    Q = rng.standard_normal((3, 1, 1, 64))
    table = np.array([[-1, 2], [0, 1], [4, -7]])
    O, LSE = cache.attend(Q, Kc, Vc, table, [3, 0, 4])
    np.testing.assert_allclose(O[0, 0, 0], Vc[2, 0, 0])                 # one key: its value
    assert (O[1:] == 0).all() and np.isneginf(LSE[1:]).all()


def test_join_of_shares():
    rng = np.random.default_rng(3)
    Kc, Vc = rng.standard_normal((2, 6, 2, 4, 64))
    Q = rng.standard_normal((1, 4, 1, 64))
    whole = cache.attend(Q, Kc, Vc, np.arange(6)[None], [24])
    shares = [cache.attend(Q, Kc, Vc, np.array([t]), [8]) for t in ([0, 3], [5, 1], [2, 4])] + [cache.attend(Q, Kc, Vc, np.array([[-1]]), [4])]
    O, LSE = cache.join(*(np.stack(x) for x in zip(*shares)))
    np.testing.assert_allclose(O, whole[0], atol=1e-12)
    np.testing.assert_allclose(LSE, whole[1], atol=1e-12)
    O, LSE = cache.join(np.full((2, 1, 1, 1, 64), np.nan), np.full((2, 1, 1, 1), -np.inf))
    assert (O == 0).all() and np.isneginf(LSE).all()


def test_append_turns_by_the_position_and_leaves_other_rows():
    rng = np.random.default_rng(4)
    K, V, Q = rng.standard_normal((3, 2, 1, 3, 64))
    f = [0.5, 0.25]
    Kc = Vc = np.zeros((2, 1, 4, 64))
    Qr, Kc, Vc = cache.append(K, V, Kc, Vc, np.array([[1], [0]]), [3, 4], counts=[1, 5], first=[100, 0], inv_freq=f, Q=Q, Qr=np.full_like(Q, 9.0))
    np.testing.assert_array_equal(Kc[1, 0, 2], cache.rotate(K[0, 0, :1], [102], f)[0])
    np.testing.assert_array_equal(Kc[0, 0, 3], cache.rotate(K[1, 0, 2:], [3], f)[0])
    assert (Kc[1, 0, [0, 1, 3]] == 0).all() and (Qr[0, 0, 1:] == 9).all() and (Qr[1] != 9).all()
    np.testing.assert_array_equal(Vc[0, 0, 1:], V[1, 0])
