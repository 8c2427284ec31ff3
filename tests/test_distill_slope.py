"""distill_slope.py against central differences of the loss, in 64 bits, without a GPU."""
import numpy as np
import pytest

import distill_slope as S

INF = float("inf")


def case(kind, vocab=9, k=3):
    rng = np.random.default_rng(5)
    z = rng.normal(size=(2, vocab)) * 2
    ids = np.array([[1, 4, 6], [8, 0, 5]])[:, :k]
    p = np.array([[0.4, 0.3, 0.1], [0.6, 0.15, 0.05]])[:, :k]
    if kind == "above one":
        p = p * 1.02 / p.sum(1, keepdims=True)
    if kind == "masked":
        keep = np.zeros((2, vocab), bool)
        np.put_along_axis(keep, ids, True, 1)
        z = np.where(keep, z, -INF)
    if kind == "lowest":
        keep = np.zeros((2, vocab), bool)
        np.put_along_axis(keep, ids, True, 1)
        z = np.where(keep, z, -3e38)
    if kind == "far":                # finite and positive, and 2^-1000 of the row all the same
        z += 100
        np.put_along_axis(z, ids, np.take_along_axis(z, ids, 1) + 900, 1)
    if kind == "whole vocabulary":
        z = z[:, :3]
        ids = np.array([[0, 2, 1], [1, 0, 2]])
    if kind == "nothing":
        p = p * 0
    if kind == "twice":
        ids = np.array([[1, 1, 6], [8, -1, 5]])
    with np.errstate(divide="ignore"):
        return z, ids, np.log(p)


@pytest.mark.parametrize("kind", ["plain", "above one", "masked", "lowest", "far", "whole vocabulary", "nothing", "twice"])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("temp", [1.0, 0.6])
def test_the_slope_is_that_of_the_loss(kind, rest, temp):
    """Error of a central difference: h^2 / 6 times the third derivative (P / T^3 at most) and 2^-52 |z| / (T h)."""
    z, ids, lp = case(kind)
    g, h = np.array([1.5, -0.75]), 1e-5
    grad = S.distill(z, ids, lp, temp, rest, g)[3]
    with np.errstate(invalid="ignore"):
        for v in range(z.shape[1]):
            up, down = z.copy(), z.copy()
            up[:, v] += h
            down[:, v] -= h
            want = (S.distill(up, ids, lp, temp, rest)[0] - S.distill(down, ids, lp, temp, rest)[0]) / (2 * h) * g
            assert (np.abs(grad[:, v] - want) <= 2 * (h * h / temp ** 3 + 2.0 ** -52 * (4 + np.abs(np.where(np.abs(z) < 1e30, z, 0)).max()) / (temp * h))).all(), v


def test_ordinary_rows_have_mass_one_and_the_others_do_not():
    for kind, rest, want in (("plain", True, 1), ("plain", False, 1), ("masked", True, 0.8), ("above one", True, 1.02), ("nothing", False, 0), ("nothing", True, 1), ("masked", False, 1)):
        z, ids, lp = case(kind)
        assert np.allclose(S.masses(z, ids, lp, 1.0, rest), want, rtol=1e-12)


def test_without_the_mass_it_is_not():
    """What draft_reference.distill gives in such rows (its gradient does not even sum to 0, as that of a function of differences of logits must)."""
    for kind, rest in (("masked", True), ("above one", True), ("nothing", False)):
        z, ids, lp = case(kind)
        assert np.abs(S.without_mass(z, ids, lp, 1.0, rest, np.ones(2))[3].sum(1)).min() > 0.01
        assert np.abs(S.distill(z, ids, lp, 1.0, rest, np.ones(2))[3].sum(1)).max() < 1e-12
