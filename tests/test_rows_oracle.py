"""The 64-bit oracle of the operators around the head's product, against plain definitions
and against differences (no GPU needed)."""
import numpy as np
import pytest

from oracle import rows_oracle as ora
from oracle.table_oracle import e4m3_table


def test_norm_of_a_plain_row():
    y, mean, rstd = ora.norm([[1.0, 3.0, 5.0, 7.0]], eps=0.0)
    assert mean[0] == 4 and np.isclose(rstd[0], 1 / np.sqrt(5))
    assert np.allclose(y, (np.array([[1, 3, 5, 7.0]]) - 4) / np.sqrt(5))
    y, mean, rstd = ora.norm([[3.0, 4.0]], weight=[2.0, 1.0], bias=[0.5, 0.0], eps=0.0, centre=False)
    assert mean[0] == 0 and np.allclose(y, [[2 * 3 / np.sqrt(12.5) + 0.5, 4 / np.sqrt(12.5)]])


@pytest.mark.parametrize("centre", [True, False])
def test_gradients_are_those_of_differences(centre):
    rng = np.random.default_rng(1)
    x, w, b = rng.standard_normal((3, 7)) + 0.4, rng.standard_normal(7), rng.standard_normal(7)
    dy = rng.standard_normal((3, 7))
    loss = lambda x, w, b: (ora.norm(x, w, b, 1e-3, centre)[0] * dy).sum()
    _, mean, rstd = ora.norm(x, w, b, 1e-3, centre)
    dx, dw, db = ora.norm_grads(dy, x, w, mean if centre else None, rstd)
    for got, at, k in ((dx, x, 0), (dw, w, 1), (db, b, 2)):
        want = np.zeros_like(at)
        for i in np.ndindex(at.shape):
            args = [x.copy(), w.copy(), b.copy()]
            args[k][i] += 1e-6
            hi = loss(*args)
            args[k][i] -= 2e-6
            want[i] = (hi - loss(*args)) / 2e-6
        assert np.abs(got - want).max() < 1e-7


def test_e4m3_blocks():
    grid = e4m3_table()
    # 448 fixes the scale at one: every value of the grid is held exactly, midpoints go to even
    x = np.zeros((1, 128))
    x[0, 0] = 448
    x[0, 1:] = grid
    codes, scales = ora.encode8(x)
    assert scales[0, 0] == 1 and np.array_equal(codes[0, 1:], np.arange(127))
    x[0, 1:127] = (grid[:-1] + grid[1:]) / 2
    x[0, 127] = -0.0
    codes, _ = ora.encode8(x)
    assert (codes[0, 1:127] % 2 == 0).all() and codes[0, 127] == 128
    # a block of 128 rows has one scale
    x = np.ones((130, 129))
    x[5, 3], x[129, 128] = 896, 4480
    codes, scales = ora.encode8(x, 128)
    assert scales.shape == (2, 2)
    assert np.array_equal(scales[0], np.float32([2, np.float32(1) / np.float32(448)]))
    assert scales[1, 1] == 10
    assert np.abs(ora.held8(x, 128)[:128, 128] - 1).max() < 1e-7
    x[0, 0] = np.nan
    held = ora.held8(x, 128)
    assert np.isnan(held[:128, :128]).all() and not np.isnan(held[128:]).any()


def test_shape_in_steps():
    z = np.array([[2.0, -2.0, 1.0, 0.0, 5.0]])
    y = ora.shape(z, 5, history=[[0, 1, 1, 4, 9, -1]], lengths=[5], prompts=[1], repetition=[2.0],
                  frequency=[0.5], presence=[0.25], bias_ids=[[3, -1, 3]],
                  bias_values=[[1.0, 7.0, 2.0]], mask=[[0b01111]])
    assert np.array_equal(y, [[1.0, -4.0 - 1.0 - 0.25, 1.0, 3.0, -np.inf]])
    y = ora.shape(z[:, :2], 40, ids=[1, 39], mask=[[0, 1 << 7]], mask_rows=[0])
    assert np.array_equal(y, [[-np.inf, -2.0]])
    assert np.array_equal(ora.shape(z, 5, mask=[[0]], mask_rows=[-1]), z)
