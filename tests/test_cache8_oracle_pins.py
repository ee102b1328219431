"""The oracle of the cache in 8 bits and of several new tokens at a time, against torch's own e4m3 and against the single token."""
import numpy as np
import torch

from oracle import cache


def test_numbers_of_e4m3_are_torchs():
    b = np.arange(256)
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(cache.from_e4m3(b), t)


def test_every_bf16_number_of_a_row_is_rounded_as_torch_rounds_it():
    """Rows whose largest element sets the power to 1: 448 and numbers below it."""
    x = torch.arange(0, 0x43E0 + 1).to(torch.int16).view(torch.bfloat16)
    x = torch.cat([x, -x]).reshape(-1, 1)
    rows = torch.cat([x, torch.full_like(x, 448.0)], 1).double().numpy()
    byte, e = cache.to_e4m3(rows)
    assert (e == 127).all()
    want = torch.from_numpy(rows).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(byte, want)


def test_powers():
    rows = np.array([[448.0, 1], [449, 1], [224, 0], [224.5, 0], [0, 0], [2.0 ** -56, 0], [1.75 * 2.0 ** -56, 0], [1.76 * 2.0 ** -56, 0], [3e38, 1],
                     [np.inf, 1], [np.nan, -3]])
    byte, e = cache.to_e4m3(rows)
    np.testing.assert_array_equal(e - 127, [0, 1, -1, 0, -64, -64, -64, -63, 120, -8, -7])
    assert byte[9, 0] == byte[10, 0] == 127 and byte[10, 1] == 128 + cache.to_e4m3(rows[10:11] * 0 + [[0, 3]])[0][0, 1]
    v = cache.from_e4m3(byte) * 2.0 ** (e - 127)[:, None]
    fine = np.isfinite(rows[:9])
    assert (np.abs(v[:9] - rows[:9])[fine] <= np.maximum(2.0 ** -4 * np.abs(rows[:9]), 2.0 ** (e[:9, None] - 127 - 10))[fine]).all()


def test_what_is_appended_is_read():
    rng = np.random.default_rng(0)
    K, V = rng.standard_normal((2, 2, 1, 3, 64))
    pools = [np.zeros((3, 1, 4, 64))] * 2 + [np.full((3, 1, 4), 255)] * 2
    table, lengths, counts = np.array([[2, 0], [1, -1]]), [5, 6], [3, 3]
    _, Kc, Vc, Ks, Vs = cache.append8(K, V, *pools, table, lengths, counts)
    got = cache.read(cache.from_e4m3(Vc) * 2.0 ** (Vs - 127.0)[..., None], table, lengths, 3, counts)
    byte, e = cache.to_e4m3(V)
    want = cache.from_e4m3(byte) * 2.0 ** (e - 127.0)[..., None]
    want[1, :, 1:] = 0                                       # slots 4 and 5 of the second sequence are not held
    np.testing.assert_array_equal(got, want)
    assert (Ks == 255).sum() == 12 - 4 and (np.abs(want[0] - V[0]) <= 2.0 ** -4 * np.abs(V[0]) + 2.0 ** -10 * 2.0 ** (e[0, ..., None] - 127)).all()


def test_a_chunk_is_its_tokens_one_by_one():
    rng = np.random.default_rng(1)
    Kc, Vc = rng.standard_normal((2, 4, 2, 4, 64))
    Q = rng.standard_normal((2, 4, 3, 64))
    table = np.array([[3, 1], [0, -1]])
    O, LSE = cache.attend_chunk(Q, Kc, Vc, table, [8, 2], [3, 2])
    for t in range(3):
        o, l = cache.attend(Q[:1, :, t:t + 1], Kc, Vc, table[:1], [6 + t])
        np.testing.assert_array_equal(O[:1, :, t:t + 1], o)
        np.testing.assert_array_equal(LSE[:1, :, t:t + 1], l)
    np.testing.assert_allclose(O[1, :, 0], np.repeat(Vc[0, :, 0], 2, 0))      # its first slot alone
    assert (O[1, :, 2] == 0).all() and np.isneginf(LSE[1, :, 2]).all()
    all_of_them = cache.attend_chunk(Q, Kc, Vc, table, [8, 2], None, causal=False)
    np.testing.assert_array_equal(all_of_them[0][:, :, 2:], cache.attend(Q[:, :, 2:], Kc, Vc, table, [8, 2])[0])
