"""The oracle of the operators on a router's logits: its gradients against differences of its own losses, in 64 bits."""
import numpy as np
import pytest

from oracle import router as R


def _difference(f, x, h=1e-5):
    """The gradient of f(x) by central differences, entry by entry."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        if x[i] == -np.inf:
            continue
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def _rows(rng, T, E, out=True):
    x = rng.normal(size=(T, E)) * 1.5
    if out:
        x[rng.random((T, E)) < 0.15] = -np.inf
        x[:, 0] = rng.normal(size=T)
        x[1] = -np.inf                                      # a row without an expert
    return x


# h^2 / 6 of the third derivative (of order 1 here) and the rounding 2^-53 |f| / h: below 1e-9 for losses of order 10
CLOSE = 1e-8


@pytest.mark.parametrize("tau", [1.0, 0.5, 3.0])
def test_logprobs_gradient(tau):
    rng = np.random.default_rng(1)
    x = _rows(rng, 6, 9)
    idx = rng.integers(-1, 10, size=(6, 4))
    idx[2] = [3, 3, 3, 0]
    idx = np.where(np.take_along_axis(x, np.clip(idx, 0, 8), 1) == -np.inf, 0, idx)        # a pick that is out has no finite log probability
    mask = np.array([1, 1, 1, 0, 1, 1])
    dl, dz, dh = rng.normal(size=(6, 4)), rng.normal(size=6), rng.normal(size=6)

    def f(v):
        logp, lse, h, _, _ = R.logprobs(v, idx, 0, tau, mask)
        return (logp * dl).sum() + (lse * dz).sum() + (h * dh).sum()

    g, size = R.logprobs_backward(x, idx, dl, dz, dh, tau, mask)
    assert np.abs(g - _difference(f, x)).max() < CLOSE and np.all(np.abs(g) <= size + 1e-12)
    assert not g[1].any() and not g[3].any()


def test_balance_gradient_and_even_spread():
    rng = np.random.default_rng(2)
    x = _rows(rng, 10, 7)
    idx = rng.integers(-1, 8, size=(10, 3))
    edges = [(0, 4), (4, 4), (4, 9)]
    mask = np.array([1, 1, 0, 1, 1, 1, 1, 1, 1, 1])
    counts, tokens, _, _ = R.balance(x, idx, edges, 0.3, mask)
    d = rng.normal(size=3)
    g, size = R.balance_backward(x, 3, edges, 0.3, counts, tokens, d, mask)

    def f(v):
        _, _, sums, _ = R.balance(v, idx, edges, 0.3, mask)
        n = np.maximum(tokens, 1).astype(float)
        return (d * 0.3 * 7 / (3 * n * n) * (counts * sums).sum(axis=1)).sum()

    assert np.abs(g[:9] - _difference(f, x)[:9]).max() < CLOSE and np.isnan(g[9]).all() and np.all(np.abs(g[:9]) <= size[:9] + 1e-12)
    even = np.zeros((8, 4))
    _, _, _, loss = R.balance(even, np.arange(16).reshape(8, 2) % 4, [(0, 8)], 0.7)
    assert abs(loss[0] - 0.7) < 1e-14


@pytest.mark.parametrize("tau", [1.0, 2.0])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient(tau, tail):
    rng = np.random.default_rng(3)
    x = _rows(rng, 7, 9)
    t = x + rng.normal(size=(7, 9)) * 0.5
    t[1] = rng.normal(size=9)
    idx = np.argsort(-t, axis=1, kind="stable")[:, :4]
    logit = np.take_along_axis(t, idx, 1)
    idx[2, 3], logit[2, 3] = idx[2, 0], logit[2, 0]         # an expert twice
    idx[4, 1] = -1                                          # an entry that is absent
    idx[5] = -1                                             # none at all
    lse = np.log(np.exp(t / tau).sum(axis=1)) if tail else None
    d = rng.normal(size=7)

    def f(v):
        return (R.distill(v, idx, logit, lse, tau) * d).sum()

    g, size = R.distill_backward(x, idx, logit, d, lse, tau)
    assert np.abs(g - _difference(f, x)).max() < CLOSE * tau * tau and np.all(np.abs(g) <= size + 1e-12)
    assert not g[1].any() and not g[5].any()
    full = np.tile(np.arange(9), (7, 1))
    assert np.abs(R.distill(x[[0, 2]], full[:2], x[[0, 2]], None, tau)).max() < 1e-14       # the same router: no divergence
