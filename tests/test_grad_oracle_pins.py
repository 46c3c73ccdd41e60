"""The fp64 gradients that kvb_scan_backward is tested against, pinned by differences of the recurrence itself, and its forward
pass by the C oracle."""
import numpy as np
import pytest

from oracle import gdn, gdn_grad


def problem(T=7, Hk=2, Hv=4, d=6, seed=0):
    rng = np.random.default_rng(seed)
    x = {"S": rng.standard_normal((Hv, d, d)), "q": rng.standard_normal((T, Hk, d)), "k": rng.standard_normal((T, Hk, d)) / np.sqrt(d),
         "v": rng.standard_normal((T, Hv, d)), "g": -rng.random((T, Hv)), "beta": rng.random((T, Hv))}
    return x, rng.standard_normal((T, Hv, d)), rng.standard_normal((Hv, d, d))


def test_forward_is_the_recurrence():
    x, _, _ = problem()
    o, _, S = gdn_grad.forward(*(x[n] for n in ("S", "q", "k", "v", "g", "beta")), 0.3)
    want, _, Sw, _ = gdn.gdn_sequence(x["S"][None], *(x[n][None] for n in ("q", "k", "v", "g", "beta")), 0.3)
    assert np.abs(o - want[0]).max() < 1e-12 and np.abs(S - Sw[0]).max() < 1e-12


@pytest.mark.parametrize("name, at", [("q", 0), ("k", 1), ("v", 2), ("g", 3), ("beta", 4), ("S", 5)])
def test_gradients_are_differences(name, at):
    """Central differences with a step of 1e-5 leave an error of the third derivative times 1e-10, and rounding of 1e-11."""
    x, dout, dS = problem(seed=at)

    def loss(y):
        o, _, S = gdn_grad.forward(*({**x, name: y}[n] for n in ("S", "q", "k", "v", "g", "beta")), 0.3)
        return (o * dout).sum() + (S * dS).sum()

    got = gdn_grad.backward(*(x[n] for n in ("S", "q", "k", "v", "g", "beta")), 0.3, dout, dS)[at]
    rng = np.random.default_rng(1)
    for _ in range(8):
        way = rng.standard_normal(x[name].shape)
        want = (loss(x[name] + 1e-5 * way) - loss(x[name] - 1e-5 * way)) / 2e-5
        assert abs((got * way).sum() - want) < 1e-7 * max(1.0, abs(want))
