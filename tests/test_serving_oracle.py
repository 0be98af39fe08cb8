"""The plain float64 definitions of the norm, cache and attention operators, checked against what fixes them:
hand-worked values, central differences and the properties of the definitions (no GPU)."""
import numpy as np
import pytest

from oracle import serving_oracle as SO


def test_norm_hand_worked():
    # mean square of (3, 4) is 12.5; gamma (1, -2)
    y = SO.rmsnorm([[3.0, 4.0]], [1.0, -2.0], 0.0)
    assert np.allclose(y, [[3 / np.sqrt(12.5), -8 / np.sqrt(12.5)]], rtol=1e-15)
    assert np.array_equal(SO.token_scale(np.array([[0.0, 0.0], [-254.0, 1.0]])), [1.0, 2.0])


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(0)
    h, gamma, dy, dh = rng.normal(size=(3, 8)), rng.normal(size=8), rng.normal(size=(3, 8)), rng.normal(size=(3, 8))
    dx, dgamma = SO.rmsnorm_bwd(dy, h, gamma, 1e-5, dh)
    loss = lambda h_, g_: (SO.rmsnorm(h_, g_, 1e-5) * dy).sum() + (h_ * dh).sum()  # noqa: E731
    eps = 1e-6
    for i in range(3):
        for j in range(8):
            e = np.zeros((3, 8))
            e[i, j] = eps
            assert abs((loss(h + e, gamma) - loss(h - e, gamma)) / (2 * eps) - dx[i, j]) < 1e-7
    for j in range(8):
        e = np.zeros(8)
        e[j] = eps
        assert abs((loss(h, gamma + e) - loss(h, gamma - e)) / (2 * eps) - dgamma[j]) < 1e-7


def test_cache_write_hand_worked():
    c = SO.Cache(3, 1, 2, 2)
    c.write([[[127.0, -63.5]]], 1, [2, 0])                   # scale 1; 63.5 rounds to the even 64
    assert c.scale[2, 0] == 1 and c.codes[2, 0, 0].tolist() == [127, -64]
    c.write([[[254.0, 2.0]], [[0.0, 0.0]]], 3, [2, 0])       # the block's scale doubles; a block of zeros has scale 1
    assert c.scale[2, 0] == 2 and c.codes[2, 0].tolist() == [[64, -32], [127, 1]]    # 63.5 -> 64
    assert c.scale[0, 0] == 1 and c.codes[0, 0, 0].tolist() == [0, 0]
    before = c.codes.copy(), c.scale.copy()
    c.write([[[254.0, 2.0]], [[0.0, 0.0]]], 3, [2, 0])       # writing the same rows again changes nothing
    assert np.array_equal(before[0], c.codes) and np.array_equal(before[1], c.scale, equal_nan=True)
    assert c.values(3, [2, 0])[:, 0].tolist() == [[128, -64], [254, 2], [0, 0]]


def test_cache_rounding_error_is_within_half_a_step():
    rng = np.random.default_rng(1)
    c = SO.Cache(8, 2, 16, 4)
    x = rng.normal(size=(50, 2, 4)).astype(np.float32)
    c.write(x, 50, [3, 1, 7, 0])
    v = c.values(50, [3, 1, 7, 0])
    step = c.scale[[3, 1, 7, 0]].astype(np.float64)[np.arange(50) // 16]
    assert (np.abs(v - x) <= 0.5001 * step[:, :, None]).all()


@pytest.mark.parametrize("window", [0, 1, 3])
def test_attention_rows_are_convex_combinations(window):
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(2, 7, 2, 4))
    q = rng.normal(size=(9, 4, 4))                           # two more rows than positions
    o, _, seen = SO.attention(q, k, v, 7, 0.5, window)
    assert seen.tolist() == [0, 0] + [min(i + 1, window or 9) for i in range(7)]
    assert (o[:2] == 0).all()
    assert np.allclose(o[2], np.repeat(v[0], 2, 0))          # the first position sees itself alone
    if window == 1:
        assert np.allclose(o[2:], np.repeat(v, 2, 1))
    same, _, _ = SO.attention(q, k, np.ones_like(v), 7, 0.5, window)
    assert np.allclose(same[2:], 1.0)


def test_cache_zeros_fix_no_scale():
    c = SO.Cache(1, 1, 4, 2)
    c.write([[[0.0, 0.0]]], 1, [0])
    c.write([[[0.25, -0.5]]], 2, [0])                        # behind zeros: as if the block started here
    assert c.scale[0, 0] == np.float32(0.5) / np.float32(127) and c.codes[0, 0].tolist()[:2] == [[0, 0], [64, -127]]
    c.write([[[127.0, 0.0]]], 3, [0])                        # 64 and -127 steps of 0.5 / 127 are less than half of one of 1
    assert c.scale[0, 0] == 1 and c.codes[0, 0].tolist()[:3] == [[0, 0], [0, 0], [127, 0]]
    c.write([[[0.25, 0.0]]], 4, [0])                         # a scale of 1 that a token does need
    assert c.scale[0, 0] == 1 and c.codes[0, 0].tolist()[3] == [0, 0]
