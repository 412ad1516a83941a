"""What pins the oracle of positions, cache and attention (oracle/attention_oracle.py) itself: properties that follow from the definitions,
and hand-worked numbers.  No GPU."""
import numpy as np
import pytest

from oracle import attention_oracle as oracle
from paper_2603_09221_amd import binding


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_keeps_lengths_and_depends_on_distance_only(layout):
    rng = np.random.default_rng(1)
    freqs, _ = binding.rope_frequencies(8)
    table = oracle.rope_table(64, freqs.numpy())
    q, k = rng.standard_normal((2, 1, 1, 12))
    def at(x, p):
        return oracle.rope(x, [p], table, layout)
    np.testing.assert_allclose(np.linalg.norm(at(q, 37)), np.linalg.norm(q), rtol=1e-14)
    np.testing.assert_allclose((at(q, 9) * at(k, 4)).sum(), (at(q, 45) * at(k, 40)).sum(), rtol=1e-12)
    np.testing.assert_array_equal(at(q, 9)[..., 8:], q[..., 8:])
    np.testing.assert_allclose(oracle.rope(at(q, 9), [9], table, layout, backward=True), q, rtol=1e-14)


def test_rotation_by_a_quarter_turn():
    table = np.array([[[0.0, 1.0], [0.0, 1.0]]])
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    np.testing.assert_array_equal(oracle.rope(x, [0], table, "half"), [[[-3.0, -4.0, 1.0, 2.0]]])
    np.testing.assert_array_equal(oracle.rope(x, [0], table, "interleaved"), [[[-2.0, 1.0, -4.0, 3.0]]])


def test_gradient_of_the_rotation_against_differences():
    rng = np.random.default_rng(2)
    table = oracle.rope_table(16, binding.rope_frequencies(6)[0].numpy(), scale=1.2)
    x, g = rng.standard_normal((2, 2, 1, 7))
    want = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        step = np.zeros_like(x)
        step[i] = 1e-5
        want[i] = ((oracle.rope(x + step, [3, 11], table) - oracle.rope(x - step, [3, 11], table)) * g).sum() / 2e-5
    np.testing.assert_allclose(oracle.rope(g, [3, 11], table, backward=True), want, atol=1e-9)


def test_codes_by_hand():
    x = np.zeros((1, 32))
    x[0, :12] = [7.0, 6.9, -5.0, 5.1, 3.5, 2.5, 1.25, 1.75, 0.25, 0.26, -0.75, -0.1]
    # the largest is 1.75 * 2^2: one exponent more, everything is halved
    codes, e = oracle.quantise(x)
    assert e[0, 0] == 128
    # 3.5 (tie of 3 and 4: the even code), 3.45, -2.5 (tie of 2 and 3: the even code), 2.55, 1.75 (tie of 1.5 and 2), 1.25, 0.625, 0.875, 0.125, 0.13, -0.375, -0.05
    assert codes[0, :12].tolist() == [6, 5, 8 + 4, 5, 4, 2, 1, 2, 0, 0, 8 + 1, 8 + 0]
    x[0, 0] = 6.9
    codes, e = oracle.quantise(x)
    assert e[0, 0] == 127 and codes[0, :4].tolist() == [7, 7, 8 + 6, 7]


def test_rounding_moves_a_number_by_at_most_half_a_step():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((200, 64)) * np.exp(rng.standard_normal((200, 1)) * 10)
    codes, e = oracle.quantise(x)
    scale = np.repeat(np.exp2(e - 127.0), 32, -1)
    y = np.abs(x) / scale
    half = np.where(y <= 2, 0.25, np.where(y <= 4, 0.5, 1.0))
    assert (np.abs(oracle.numbers(codes, e) - x) <= half * scale).all()
    again = oracle.numbers(*oracle.quantise(oracle.numbers(codes, e)))
    assert (np.abs(again - oracle.numbers(codes, e)) <= half * scale).all()


def test_blocks_without_finite_numbers_are_nan():
    x = np.ones((3, 64))
    x[0, 5], x[1, 40], x[2, 0] = np.nan, np.inf, 0.0
    v = oracle.numbers(*oracle.quantise(x))
    assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:]).all() and not np.isnan(v[2]).any()
    assert not np.isnan(v[0, 32:]).any() and not np.isnan(v[1, :32]).any()


def test_attention_over_equal_keys_is_the_mean_of_what_is_seen():
    rng = np.random.default_rng(4)
    k, v = np.ones((32, 1, 64)), rng.standard_normal((32, 1, 64))
    q = rng.standard_normal((3, 2, 64))
    table = np.array([[1, 0]])
    out, lse, _ = oracle.attention(q, k, v, table, [20], [0, 3], 16, 2, 0.5)
    order = np.concatenate([np.arange(16, 32), np.arange(16)])
    for i, n in enumerate((18, 19, 20)):
        np.testing.assert_allclose(out[i], np.broadcast_to(v[order[:n], 0].mean(0), (2, 64)))
        np.testing.assert_allclose(lse[i], 0.5 * q[i].sum(-1) + np.log(n))
    out, lse, _ = oracle.attention(q, k, v, table, [20], [0, 3], 16, 2, 0.5, window=4)
    np.testing.assert_allclose(out[2, 0], v[order[16:20], 0].mean(0))
    out, lse, _ = oracle.attention(q, k, v, table, [2], [0, 3], 16, 2, 0.5)   # the first of the three sees nothing
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all()


def test_frequencies_for_longer_contexts():
    plain, one = binding.rope_frequencies(64)
    assert one == 1.0 and plain[0] == 1.0
    np.testing.assert_allclose(plain[-1], 10000.0 ** (-62 / 64))
    linear, _ = binding.rope_frequencies(64, scaling="linear", factor=4)
    np.testing.assert_allclose(linear, plain / 4)
    grown, _ = binding.rope_frequencies(64, scaling="base", factor=4)
    np.testing.assert_allclose([grown[0], grown[-1]], [plain[0], plain[-1] / 4])
    bands, scale = binding.rope_frequencies(64, scaling="bands", factor=4, trained=4096)
    turns = 4096 * plain / (2 * np.pi)
    fast, slow = turns > 45, turns < 0.7    # (the bands' ends are whole indices)
    assert fast.any() and slow.any()
    np.testing.assert_allclose(bands[fast], plain[fast])
    np.testing.assert_allclose(bands[slow], plain[slow] / 4)
    assert ((bands <= plain) & (bands >= plain / 4 * (1 - 1e-12))).all() and abs(scale - (0.1 * np.log(4) + 1)) < 1e-12
    for bad in (dict(rot=7), dict(rot=8, scaling="other"), dict(rot=8, scaling="bands", factor=2), dict(rot=8, factor=0.5)):
        with pytest.raises(ValueError):
            binding.rope_frequencies(**bad)
