"""The oracle's distillation gradient against difference quotients where the list's
probabilities and the mass beside them do not sum to one."""
import numpy as np
import pytest

from oracle import scores as orc

V = 24


def quotient(l, ids, val, tail, tau, h=1e-5):
    """Central differences of the loss in the finite logits (0 at the others, whose
    probability is 0 whatever is added to them)."""
    g = np.zeros(V)
    for i in np.where(np.isfinite(l))[0]:
        a, b = l.copy(), l.copy()
        a[i] += h
        b[i] -= h
        g[i] = (orc.distill(a, ids, val, tail, tau)[0] - orc.distill(b, ids, val, tail, tau)[0]) / (2 * h)
    return g


def case(masked, whole):
    rng = np.random.default_rng(7)
    l, t = rng.normal(0, 2, V), rng.normal(0, 2, V)
    ids = list(range(V)) if whole else [int(i) for i in np.argsort(-t)[:7]]
    if masked:
        l[[i for i in range(V) if i not in ids]] = -np.inf
    return l, ids, t


@pytest.mark.parametrize("tau", [1.0, 0.5, 2.0])
@pytest.mark.parametrize("masked,whole", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("mass", [0.3, 0.85, 1.0, 1.004, 1.27])
def test_gradient_of_lists_of_any_mass(mass, masked, whole, tau):
    l, ids, t = case(masked, whole)
    val = orc.log_softmax(t, tau)[ids]
    val += np.log(mass / np.sum(np.exp(val)))
    grad = orc.distill(l, ids, val, True, tau)[1]
    # A central difference is off by h^2 f''' / 6 (third derivatives below 2 mass / tau) and by
    # rounding, 2^-52 |f| / h with |f| below 40.
    assert np.allclose(grad, quotient(l, ids, val, True, tau), rtol=0, atol=2e-9)
    # The loss does not change when every logit moves by the same amount: at most V terms
    # of 2 tau mass, each with a few roundings of 2^-53.
    assert abs(np.sum(grad)) < 1e-13


@pytest.mark.parametrize("masked", [False, True])
def test_gradient_without_a_tail(masked):
    l, ids, t = case(masked, False)
    grad = orc.distill(l, ids, t[ids], False, 1.5)[1]
    assert np.allclose(grad, quotient(l, ids, t[ids], False, 1.5), rtol=0, atol=2e-9)
    assert abs(np.sum(grad)) < 1e-13
