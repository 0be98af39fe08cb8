"""The plain float64 definitions of the head norm and rotation and the sequential one of the block tables, checked against
what fixes them: hand-worked values, central differences and properties (no GPU)."""
import numpy as np
import pytest

from oracle import serving_oracle as SO


def test_rotation_hand_worked():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    half = np.pi / 2
    assert np.allclose(SO.rotate(x, [1], [half, 0.0]), [[[-3, 2, 1, 4, 9]]])            # pairs (0, 2), (1, 3); 4 passes
    assert np.allclose(SO.rotate(x, [1], [half, 0.0], neighbours=True), [[[-2, 1, 3, 4, 9]]])
    assert np.allclose(SO.rotate(x, [2], [half, half / 2]), [[[-1, -4, -3, 2, 9]]])
    assert np.allclose(SO.rotate(SO.rotate(x, [5], [0.3, 2.0]), [5], [0.3, 2.0], back=True), x)


@pytest.mark.parametrize("neighbours", [False, True])
def test_scores_depend_on_the_distance_alone(neighbours):
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(2, 1, 1, 8))
    freq = [1.0, 0.2, 0.03, 0.0]
    at = lambda p, r: float((SO.rotate(q, [p], freq, neighbours) * SO.rotate(k, [r], freq, neighbours)).sum())  # noqa: E731
    assert np.allclose([at(7 + s, 3 + s) for s in (0, 1, 1000, 123456)], at(7, 3), rtol=1e-9)


@pytest.mark.parametrize("neighbours,norm", [(False, True), (True, True), (False, False)])
def test_gradient_against_differences(neighbours, norm):
    rng = np.random.default_rng(1)
    x, dy = rng.normal(size=(2, 3, 2, 6))
    gamma = rng.normal(size=6) if norm else None
    pos, freq = [0, 5, 77], [1.0, 0.1]
    dx, dg = SO.head_norm_rope_bwd(dy, x, gamma, pos, freq, 1e-3, neighbours)
    loss = lambda x_, g_: (SO.head_norm_rope(x_, g_, pos, freq, 1e-3, neighbours) * dy).sum()  # noqa: E731
    for i in np.ndindex(x.shape):
        e = np.zeros(x.shape)
        e[i] = 1e-6
        assert abs((loss(x + e, gamma) - loss(x - e, gamma)) / 2e-6 - dx[i]) < 1e-7
    for i in range(6 if norm else 0):
        e = np.zeros(6)
        e[i] = 1e-6
        assert abs((loss(x, gamma + e) - loss(x, gamma - e)) / 2e-6 - dg[i]) < 1e-7


def test_blocks_hand_worked():
    b = SO.Blocks([[-1, -1, -1], [50, -1, -1]], [10, 11, 12, 13, -1], 4, [0, 3], 2, 0)
    b.len[1] = 1
    seen, start, pos, slot, bad = b.extend([3, 2], 6)
    assert (seen, start, pos, bad) == ([3, 3], [0, 3, 5], [0, 1, 2, 1, 2, -1], False)
    assert b.table.tolist() == [[13, 12, -1], [50, 11, -1]] and b.free == 1
    assert slot == [26, 27, 24, 101, 22, -1]
    assert not b.truncate([2, 3]) and b.free == 2 and b.free_ids[:2].tolist() == [10, 12] and b.len == [2, 3]
    seen, start, pos, slot, bad = b.extend([-2, 4], 6)        # four more tokens need one column beyond the table
    assert bad and seen == [0, 0] and pos == [-1] * 6 and start == [0, 2, 6] and b.len == [2, 3] and b.free == 2


def test_blocks_are_never_shared():
    rng = np.random.default_rng(2)
    b = SO.Blocks(np.full((9, 40), -1), rng.permutation(100), 100, [0] * 9, 4, 0)
    for _ in range(200):
        b.extend(rng.integers(-1, 9, 9), 80)
        held = [i for row, n in zip(b.table, b.len) for i in row[:-(-n // 4)]]
        assert sorted(held + b.free_ids[:b.free].tolist()) == list(range(100))
        b.truncate([n - int(rng.integers(0, 7)) if rng.random() < 0.9 else 0 for n in b.len])
