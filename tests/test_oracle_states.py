"""The definition of states in 8 bits that are rounded at random: its random numbers, its codes, and what they are on average."""
import numpy as np
import pytest

from oracle import operators_oracle as orc


def test_random_shares():
    n, step = 256 * 3 + 9, (5 << 32) + 77
    for signed in (False, True):
        share = orc.state_random(n, signed, step, 3)
        for i in (0, 5, 127, 128, 255, 256, 700, n - 1):
            e = i % 256
            word = orc.philox4x32_10((32 * 3 + e % 128 // 4, i // 256, 77, 5), (0, 0))[e % 4]
            half = word >> 16 if (e < 128) == signed else word & 0xFFFF
            assert share[i] == (half + 0.5) / 65536
    assert not np.array_equal(orc.state_random(n, True, step, 3), orc.state_random(n, True, step + 1, 3))
    assert not np.array_equal(orc.state_random(n, True, step, 3), orc.state_random(n, True, step, 4))
    big = orc.state_random(256 * 40, False, 9)
    assert 0 < big.min() and big.max() < 1 and abs(big.mean() - 0.5) <= 6 * 12 ** -0.5 / big.size ** 0.5


@pytest.mark.parametrize("signed", [False, True])
def test_codes_are_neighbours_and_right_on_average(signed):
    x = np.repeat((1.3 + np.arange(8.0)) * 10.0 ** -np.arange(8.0), 32)        # a block of 8 values, 32 times each
    if signed:
        x[::2] *= -1
    table = orc.state_table(128 if signed else 256)
    sums, draws = np.zeros(256), 400
    for t in range(draws):
        codes, scales = orc.state_encode_at_random(x, signed, 33 + t)
        got = orc.state_decode(codes, scales, signed)
        a, low = np.abs(x) / scales[0], np.searchsorted(table, np.abs(x) / scales[0], side="right") - 1
        high = np.minimum(low + 1, table.size - 1)
        c = codes.astype(int) % 128 if signed else codes.astype(int)
        assert ((c == low) | (c == high)).all() and (got * x >= 0).all()
        sums += got
    step = np.where(high > low, table[high] - table[low], 0) * scales[0]
    # 32 draws of each value a time; a rounding's standard deviation is half a step at most, and its probability is good to 2^-17;
    # the largest value becomes the last code times an fp32 scale, half a step of which is 2^-24 of it
    mean = (sums / draws).reshape(8, 16, 2).mean(axis=1)
    x, step = x.reshape(8, 16, 2)[:, 0], step.reshape(8, 16, 2)[:, 0]
    assert (np.abs(mean - x) <= step * (6 * 0.5 / (16 * draws) ** 0.5 + 2.0 ** -17) + 2.0 ** -24 * np.abs(x)).all()


def test_values_of_the_table_stay():
    for signed in (False, True):
        table = orc.state_table(128 if signed else 256)
        x = np.resize(table, 256)
        codes, scales = orc.state_encode_at_random(x, signed, 1000)
        assert scales[0] == 1.0 and np.array_equal(codes, np.resize(np.arange(table.size), 256))


def test_a_second_moment_follows_where_the_nearest_code_does_not():
    """Gradients that fall to a tenth, beta2 = 0.999: 3,000 steps later the mean of v is the exact one's (its standard deviation over
    512 elements is below a tenth of it), and the nearest codes' ten times that."""
    n, beta = 512, 0.999
    gen = np.random.default_rng(2)
    v, near, random = np.zeros(n), np.zeros(n), np.zeros(n)
    falls = np.arange(n) % 2 == 0
    for t in range(1, 3501):
        g2 = (gen.standard_normal(n) * np.where(falls & (t > 500), 0.1, 1.0)) ** 2
        move = lambda x: beta * x + (1 - beta) * g2
        v, near = move(v), orc.state_decode(*orc.state_encode(move(near), False), False)
        code = orc.state_encode_at_random(move(random), False, t) if t > 32 else orc.state_encode(move(random), False)
        random = orc.state_decode(*code, False)
    v, near, random = (x[falls].mean() for x in (v, near, random))
    assert abs(random - v) <= 0.6 * v and near > 8 * v
