"""The operators on a router's logits against their formulas in 64 bits (oracle/router.py).

Tolerances, with u = 2^-24, Z the row's largest |z| (and |t_logit / tau|, |t_lse| where a teacher is read):
  z = logit * (1/tau) is off by at most 2 u Z, t = z - top by 5 u Z, e^t by (5 Z + 2.5 |t| + 4) u of itself, and the sum of at most 1024 terms (22
  additions deep) by (5 Z + 2.5 sum p|t| + 26) u with sum p|t| <= log(E) <= 7:  the relative error of p is below
      delta = (10 Z + 2.5 |t| + 70) u,
  that of a log probability absolutely the same, its own rounding (1 + |logp|) u on top.  Sums of k terms add k u of their magnitude.
A gradient's tolerance is delta times the sum of the magnitudes that the formula adds up (the oracle returns it), plus half a step of its type:
eps(type) / 2 of the value, and half the smallest subnormal.
"""
import numpy as np
import pytest
import torch

from oracle import router as R

pytestmark = pytest.mark.gpu

rs = pytest.importorskip("paper_2510_19262_amd")

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_SUBNORMAL = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}       # fp32: below the normal range may be flushed


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def _logits(rng, T, E, dtype, gap=0, shift=0, out=0.0, scale=2.0):
    """A device view of [T][E] logits in rows of E + gap places that starts `shift` places into its memory, and its values in 64 bits."""
    x = rng.normal(size=(T, E)) * scale
    if out:
        gone = rng.random((T, E)) < out
        gone[np.arange(T), rng.integers(0, E, T)] = False
        x[gone] = -np.inf
    memory = torch.full((T * (E + gap) + shift,), float("nan"), dtype=dtype, device=DEV)         # what lies between the rows is not to be used
    view = memory[shift:].view(T, E + gap)[:, :E] if T else memory[:0].view(0, E)
    view.copy_(_dev(x).to(dtype))
    return view, view.double().cpu().numpy()


def _mask(rng, T, share=0.2):
    m = (rng.random(T) >= share).astype(np.uint8)
    return _dev(m), m


def _picks(rng, T, E, k, strange=True):
    """k experts a row, some of them twice, some outside [0, E)."""
    idx = rng.integers(0, E, size=(T, k))
    if strange and T:
        idx[rng.random((T, k)) < 0.05] = -1
        idx[rng.random((T, k)) < 0.03] = E
        idx[rng.random((T, k)) < 0.01] = 2 ** 31 - 1
        idx[T // 2] = idx[T // 2, 0]                        # one expert in every slot
    return _dev(idx.astype(np.int32)), idx


def _delta(x, tau, *more):
    """delta without its part in |t|, per row."""
    z = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=1) / tau
    for m in more:
        z = np.maximum(z, m)
    return (10 * z + 70) * U


def _t(x, tau):
    top = np.where(np.isfinite(x), x, -np.inf).max(axis=1, keepdims=True)
    return np.where(np.isfinite(x), top - np.where(np.isfinite(x), x, 0.0), 0.0) / tau


def _near(got, want, tol, what):
    got = got.double().cpu().numpy()
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    tol = np.broadcast_to(tol, want.shape)
    bad = ~(np.abs(got - np.where(fine, want, 0.0)) <= tol) & fine
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, e.g. at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}, tolerance {tol[bad][0]}"


def _gradient_near(got, want, size, x, tau, dtype, k, delta, what):
    tol = size * (delta[:, None] + (2.5 * _t(x, tau) + k) * U) + np.abs(want) * torch.finfo(dtype).eps / 2 + HALF_SUBNORMAL[dtype]
    _near(got, want, tol, what)


SHAPES = [  # rows, experts, picks, alternatives, type, gap, shift, temperature, masked, out
    (1, 1, 1, 1, "fp32", 0, 0, 1.0, False, 0.0),
    (1, 256, 8, 8, "fp32", 0, 0, 1.0, False, 0.0),
    (2, 2, 2, 2, "bf16", 0, 0, 0.5, False, 0.0),
    (65, 3, 1, 3, "fp32", 0, 0, 1.0, True, 0.0),
    (257, 4, 2, 4, "fp32", 0, 0, 1.0, True, 0.3),
    (130, 5, 2, 2, "fp16", 3, 1, 1.0, False, 0.3),
    (1000, 8, 2, 8, "fp32", 0, 0, 1.0, False, 0.0),
    (1025, 8, 2, 2, "bf16", 0, 0, 2.0, True, 0.2),
    (511, 8, 8, 0, "fp32", 4, 0, 1.0, True, 0.2),
    (333, 9, 3, 9, "fp32", 0, 0, 1.0, False, 0.0),
    (200, 12, 4, 3, "fp16", 0, 0, 1.0, False, 0.2),
    (640, 16, 4, 16, "fp32", 0, 0, 1.0, True, 0.0),
    (100, 16, 16, 4, "bf16", 8, 4, 1.0, True, 0.0),
    (300, 31, 5, 31, "fp32", 1, 0, 1.0, True, 0.1),
    (300, 32, 8, 8, "fp16", 0, 0, 0.7, False, 0.0),
    (301, 36, 6, 6, "fp32", 0, 0, 1.0, False, 0.4),
    (1023, 60, 6, 4, "fp16", 4, 0, 1.0, True, 0.1),
    (777, 61, 4, 5, "fp32", 0, 0, 1.0, True, 0.0),
    (999, 64, 6, 8, "bf16", 0, 0, 1.0, False, 0.0),
    (500, 64, 64, 64, "fp32", 0, 4, 1.0, True, 0.2),
    (129, 65, 8, 8, "bf16", 0, 0, 1.0, False, 0.0),
    (400, 96, 8, 16, "fp32", 32, 0, 1.0, False, 0.1),
    (400, 128, 8, 8, "fp16", 0, 0, 1.0, True, 0.0),
    (64, 160, 100, 9, "fp32", 0, 0, 1.0, True, 0.0),
    (200, 192, 8, 8, "fp32", 0, 0, 1.0, False, 0.0),
    (1003, 256, 8, 8, "fp32", 0, 0, 1.0, True, 0.2),
    (300, 256, 8, 4, "bf16", 8, 8, 4.0, False, 0.0),
    (100, 256, 16, 33, "fp16", 0, 1, 1.0, False, 0.0),
    (99, 257, 8, 8, "fp32", 0, 0, 1.0, True, 0.0),
    (150, 512, 10, 8, "fp32", 0, 0, 1.0, True, 0.0),
    (70, 512, 8, 20, "bf16", 0, 0, 1.0, False, 0.1),
    (33, 513, 8, 8, "fp16", 0, 0, 1.0, False, 0.0),
    (64, 1000, 8, 8, "fp32", 0, 0, 1.0, True, 0.3),
    (60, 1023, 12, 64, "bf16", 1, 0, 1.0, False, 0.0),
    (128, 1024, 16, 8, "fp32", 0, 0, 1.0, False, 0.0),
    (17, 1024, 1024, 5, "fp16", 0, 0, 1.0, True, 0.0),
]


@pytest.mark.parametrize("T,E,k,m,dtype,gap,shift,tau,masked,out", SHAPES)
def test_logprobs(T, E, k, m, dtype, gap, shift, tau, masked, out):
    rng = np.random.default_rng(T * 7919 + E)
    dtype = TYPES[dtype]
    xt, x = _logits(rng, T, E, dtype, gap, shift, out)
    it, idx = _picks(rng, T, E, k)
    mt, mask = _mask(rng, T) if masked else (None, None)
    if masked:
        xt[mt == 0] = float("nan")                          # not to be read into anything
        x = np.where(mask[:, None] != 0, x, 0.0)
    logp, lse, entropy, alt_idx, alt_logp = rs.route_logprobs(xt, it, alternatives=m, temperature=tau, row_mask=mt)
    wp, wl, wh, wi, wa = R.logprobs(x, idx, m, tau, mask)
    delta = _delta(x, tau)
    _near(logp, wp, delta[:, None] + (1 + np.where(np.isfinite(wp), np.abs(wp), 0.0)) * U, "logp")
    _near(lse, wl, delta + (1 + np.abs(wl)) * U, "lse")
    # the two parts of the entropy: log total and dot / total, whose terms e^t t carry (5 Z + 2.5|t| + 6) u each
    _near(entropy, wh, delta * (2 + np.abs(wh)) + 20 * U, "entropy")
    if m:
        np.testing.assert_array_equal(alt_idx.cpu().numpy(), wi)
        _near(alt_logp, wa, delta[:, None] + (1 + np.where(np.isfinite(wa), np.abs(wa), 0.0)) * U, "alt_logp")
    else:
        assert alt_idx is None and alt_logp is None

    g, gz, gh = (rng.normal(size=s).astype(np.float32) for s in ((T, k), T, T))
    for parts in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
        a, b, c = (v * np.float32(p) for v, p in zip((g, gz, gh), parts))
        place = torch.full((T, E + 2 * gap), 7.0, dtype=dtype, device=DEV)
        d = rs.route_logprobs_backward(xt, it, *(_dev(v) if p else None for v, p in zip((a, b, c), parts)), temperature=tau, row_mask=mt,
                                       out=place[:, :E])
        want, size = R.logprobs_backward(x, idx, a.astype(float), b.astype(float), c.astype(float), tau, mask)
        _gradient_near(d, want, size, x, tau, dtype, k, 3 * delta, f"gradient of {parts}")
        assert bool((place[:, E:] == 7.0).all())            # between the rows
    start = rng.normal(size=(T, E)).astype(np.float32)
    at = _dev(start).to(dtype)
    was = at.double().cpu().numpy()
    rs.route_logprobs_backward(xt, it, _dev(g), _dev(gz), _dev(gh), temperature=tau, row_mask=mt, accumulate=True, out=at)
    want, size = R.logprobs_backward(x, idx, g.astype(float), gz.astype(float), gh.astype(float), tau, mask)
    tol = size * (3 * delta[:, None] + (2.5 * _t(x, tau) + k) * U) + np.abs(was + want) * torch.finfo(dtype).eps / 2 + HALF_SUBNORMAL[dtype] + np.abs(was) * U
    _near(at, was + want, tol, "accumulated")


@pytest.mark.parametrize("T,E,k,m,dtype,gap,shift,tau,masked,out", SHAPES)
@pytest.mark.parametrize("ragged", [False, True])
def test_balance(T, E, k, m, dtype, gap, shift, tau, masked, out, ragged):
    rng = np.random.default_rng(T * 104729 + E)
    dtype = TYPES[dtype]
    xt, x = _logits(rng, T, E, dtype, gap, shift, out)
    if T > 3:
        x[3] = -np.inf                                      # a row without an expert does not count
        xt[3] = -float("inf")
    it, idx = _picks(rng, T, E, k)
    mt, mask = _mask(rng, T, 0.3) if masked else (None, None)
    if masked:
        xt[mt == 0] = float("nan")
        x = np.where(mask[:, None] != 0, x, 0.0)
    if ragged:                                              # empty groups, rows before the first and behind the last one
        cuts = np.sort(rng.integers(0, T + 1, size=9))
        cuts[4] = cuts[3]
        off, groups = _dev(cuts), 8
        edges = list(zip(cuts[:-1], cuts[1:]))
    else:
        groups = next(g for g in (7, 5, 4, 3, 2, 1) if T % g == 0)
        off, edges = None, [(i * (T // groups), (i + 1) * (T // groups)) for i in range(groups)]
    counts, tokens, sums, loss = rs.route_balance(xt, it, groups=groups, group_off=off, coef=0.25, row_mask=mt)
    wc, wn, ws, wl = R.balance(x, idx, edges, 0.25, mask)
    np.testing.assert_array_equal(counts.cpu().numpy(), wc)
    np.testing.assert_array_equal(tokens.cpu().numpy(), wn)
    # a column's sum: every term off by delta + 2.5 |t| u with p |t| <= 1/e, and as many additions in fp32 as rows at most
    worst = _delta(x, 1.0).max() + T * U
    _near(sums, ws, worst * ws + 2 * T * U, "prob_sum")
    share = 0.25 * E / (k * np.maximum(wn, 1.0) ** 2) * wc.sum(axis=1)
    _near(loss, wl, wl * (worst + 2 * U) + share * 2 * T * U, "loss")

    d_loss = rng.normal(size=groups).astype(np.float32)
    place = torch.full((T, E + gap), 7.0, dtype=dtype, device=DEV)
    d = rs.route_balance_backward(xt, k, counts, tokens, _dev(d_loss), group_off=off, coef=0.25, row_mask=mt, out=place[:, :E])
    want, size = R.balance_backward(x, k, edges, 0.25, wc, wn, d_loss.astype(float), mask)
    none = np.isnan(want)
    assert bool((d[_dev(none)] == 7.0).all()) and bool((place[:, E:] == 7.0).all())             # rows of no group, between the rows
    _gradient_near(torch.where(_dev(none), torch.zeros_like(d), d), np.where(none, 0.0, want), size, x, 1.0, dtype, 8, 3 * _delta(x, 1.0), "gradient")
    at = d.clone()
    was = at.double().cpu().numpy()
    rs.route_balance_backward(xt, k, counts, tokens, _dev(d_loss), group_off=off, coef=0.25, row_mask=mt, accumulate=True, out=at)
    want = np.where(none, 0.0, want)
    tol = size * (3 * _delta(x, 1.0)[:, None] + (2.5 * _t(x, 1.0) + 8) * U) + np.abs(was + want) * torch.finfo(dtype).eps / 2 + HALF_SUBNORMAL[dtype] + np.abs(was) * U
    _near(at, was + want, tol, "accumulated")


def _teacher(rng, x, K, tail, tau, near=0.5):
    T, E = x.shape
    t = np.where(np.isfinite(x), x, -3.0) + rng.normal(size=(T, E)) * near
    idx = np.argsort(-t, axis=1, kind="stable")[:, :K]
    logit = np.take_along_axis(t, idx, 1).astype(np.float32)
    lse = np.log(np.exp((t - t.max(axis=1, keepdims=True)) / tau).sum(axis=1)) + t.max(axis=1) / tau if tail else None
    return idx, logit, None if lse is None else lse.astype(np.float32)


@pytest.mark.parametrize("T,E,k,m,dtype,gap,shift,tau,masked,out", SHAPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("strange", [False, True])
def test_distill(T, E, k, m, dtype, gap, shift, tau, masked, out, tail, strange):
    rng = np.random.default_rng(T * 31 + E * 7 + tail)
    dtype = TYPES[dtype]
    K = min(64, max(k, m))
    xt, x = _logits(rng, T, E, dtype, gap, shift, 0.0 if not strange else out)
    mt, mask = _mask(rng, T) if masked else (None, None)
    idx, logit, lse = _teacher(rng, x, K, tail, tau)
    if strange:
        gone = np.take_along_axis(x, idx, 1) == -np.inf      # an expert that is out here and listed there would be +infinity: its own test
        idx[gone] = -1
        idx[rng.random(idx.shape) < 0.05] = -1
        idx[rng.random(idx.shape) < 0.03] = E
        logit[rng.random(idx.shape) < 0.05] = -np.inf
        if K > 1:
            idx[T // 3, K - 1] = idx[T // 3, 0]             # twice, and in every place
            idx[T // 2] = idx[T // 2, 0]
        idx[T // 4] = -1                                    # an empty list
        logit[idx < 0] = np.nan                             # not to be read into anything
    if masked:
        xt[mt == 0] = float("nan")
        x = np.where(mask[:, None] != 0, x, 0.0)
    args = (_dev(idx.astype(np.int32)), _dev(logit))
    lt = None if lse is None else _dev(lse)
    loss = rs.route_distill(xt, *args, lt, temperature=tau, row_mask=mt)
    clean = np.where(idx < 0, 0.0, logit).astype(float)
    l64 = None if lse is None else lse.astype(float)
    want = R.distill(x, idx, clean, l64, tau, mask)
    o = R.distill_terms(x, idx, clean, l64, tau, mask)
    p = np.where(o["good"], np.take_along_axis(o["p"], o["at"], 1), 0.0)
    d = np.abs(np.where(o["good"], np.log(np.maximum(p, 1e-300)) - (o["u"] - o["log_mass"][:, None]), 0.0))
    more = [np.where(np.isfinite(clean), np.abs(clean), 0.0).max(axis=1) / tau] + ([np.abs(lse)] if tail else [])
    delta = 2 * _delta(x, tau, *more) + 2.5 * U * np.where(o["good"], _t(x, tau)[np.arange(T)[:, None], o["at"]], 0.0).max(axis=1)
    # the terms q (e^d - 1 - d) move by |p - q| for an error delta of d, and are sums of p, q and q d where d is large; the rest by |p_r - q_r| / p_r for the
    # error delta (Q + P) of p_r - q_r, or by p_r and Q themselves
    gap_ = np.abs(o["q"].sum(axis=1) - p.sum(axis=1))
    P = p.sum(axis=1)
    large = np.where(d > 0.25, p + o["q"] * (1 + d), 0.0).sum(axis=1)
    rest = np.where(o["rest_q"] > 0, gap_ / np.maximum(o["rest_p"], 1e-300) * (o["mass"] + P), o["rest_p"] + (o["mass"] if tail else 0.0))
    tol = tau * tau * delta * (np.abs(p - o["q"]).sum(axis=1) + large + rest + P * strange) + np.abs(want) * 64 * U + 2.0 ** -100
    _near(loss, want, tol, "loss")

    g = rng.normal(size=T).astype(np.float32)
    place = torch.full((T, E + gap), 7.0, dtype=dtype, device=DEV)
    got = rs.route_distill_backward(xt, *args, _dev(g), lt, temperature=tau, row_mask=mt, out=place[:, :E])
    wd, size = R.distill_backward(x, idx, clean, g.astype(float), l64, tau, mask)
    # outside the list p_e (p_r - q_r) / p_r: the error delta (Q + P) of p_r - q_r, over p_r
    size = size + np.abs(tau * g)[:, None] * o["p"] * np.where(o["rest_q"] > 0, (o["mass"] + P) / np.maximum(o["rest_p"], 1e-300), 0.0)[:, None]
    size = np.where(o["live"][:, None], size, 0.0)
    _gradient_near(got, wd, size, x, tau, dtype, K, 2 * delta, "gradient")
    assert bool((place[:, E:] == 7.0).all())
    at = got.clone()
    was = at.double().cpu().numpy()
    rs.route_distill_backward(xt, *args, _dev(g), lt, temperature=tau, row_mask=mt, accumulate=True, out=at)
    tol = size * (2 * delta[:, None] + (2.5 * _t(x, tau) + K) * U) + np.abs(was + wd) * torch.finfo(dtype).eps / 2 + HALF_SUBNORMAL[dtype] + np.abs(was) * U
    _near(at, was + wd, tol, "accumulated")


# ------------------------------------------------------------------------------------------------ values at the edge
@pytest.mark.parametrize("E", [8, 60, 64, 256, 1024])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_strange_values(E, dtype):
    """Infinities, NaN, the type's lowest and largest values: each in a row of its own, and no row reaches another."""
    dtype = TYPES[dtype]
    low, inf = torch.finfo(dtype).min, float("inf")
    x = torch.randn((12, E), device=DEV).to(dtype)
    x[1] = -inf                                             # nothing left
    x[2, 1:] = -inf                                         # one expert left
    x[3] = low                                              # a mask that uses the lowest value on all of them ...
    x[4, 1:] = low                                          # ... or on all but one
    x[5, 3] = float("nan")
    x[6, 2] = inf
    x[7] = float("nan")
    x[8] = -low
    x[9, 0] = -0.0
    x[9, 1] = 0.0
    idx = torch.tensor([[0, 1]] * 12, dtype=torch.int32, device=DEV)
    logp, lse, entropy, alt_idx, alt_logp = rs.route_logprobs(x, idx, alternatives=3)
    logp, lse, entropy, ai, al = (v.double().cpu().numpy() for v in (logp, lse, entropy, alt_idx, alt_logp))
    assert (logp[1] == 0).all() and lse[1] == 0 and entropy[1] == 0 and (ai[1] == -1).all() and (al[1] == 0).all()
    assert logp[2, 0] == 0 and logp[2, 1] == -inf and entropy[2] == 0 and list(ai[2]) == [0, -1, -1] and al[2, 0] == 0 and (al[2, 1:] == -inf).all()
    for r in (3, 8):                                        # equal logits: even, however large
        assert np.abs(logp[r] + np.log(E)).max() < 8 * 8 * U and abs(entropy[r] - np.log(E)) < 16 * 8 * U and list(ai[r]) == [0, 1, 2]
    assert logp[4, 0] == 0 and entropy[4] == 0 and list(ai[4]) == [0, 1, 2]
    for r in (5, 6, 7):
        assert np.isnan(logp[r]).all() and np.isnan(lse[r]) and np.isnan(entropy[r])
        assert ((ai[r] >= -1) & (ai[r] < E)).all()
    for r in (0, 9, 10, 11):
        assert np.isfinite(logp[r]).all() and np.isfinite(entropy[r])
    one = torch.ones(12, device=DEV)
    for g in (rs.route_logprobs_backward(x, idx, torch.ones((12, 2), device=DEV), one, one),
              rs.route_distill_backward(x, idx, torch.zeros((12, 2), device=DEV), one),
              rs.route_distill_backward(x, idx, torch.zeros((12, 2), device=DEV), one, torch.full((12,), 3.0, device=DEV)),
              rs.route_balance_backward(x, 2, torch.arange(E, device=DEV).view(1, E), torch.full((1,), 12, device=DEV), one[:1])):
        g = g.double().cpu().numpy()
        assert (g[1] == 0).all()
        for r in (5, 6, 7):
            assert np.isnan(g[r]).all()
        assert np.isfinite(np.delete(g, (5, 6, 7), axis=0)).all()
    loss = rs.route_distill(x, idx, torch.zeros((12, 2), device=DEV)).cpu().numpy()
    assert loss[1] == 0 and loss[2] == inf and np.isnan(loss[[5, 6, 7]]).all() and np.isfinite(loss[[0, 3, 8, 9, 10, 11]]).all()
    off = torch.tensor([0, 5, 8, 12], device=DEV)
    counts, tokens, sums, bl = (v.double().cpu().numpy() for v in rs.route_balance(x, idx, group_off=off))
    assert list(tokens) == [4, 3, 4] and np.isfinite(sums[[0, 2]]).all() and np.isnan(sums[1]).all()
    assert np.isfinite(bl[[0, 2]]).all() and np.isnan(bl[1]) and list(counts[0, :3]) == [4, 4, 0]
    assert abs(sums[0].sum() - 4) < 1e-5 and abs(sums[2].sum() - 4) < 1e-5


def test_teacher_equal_to_the_student_costs_nothing():
    """Second-order accuracy: where p is near q the loss is as small as it is, not the rounding of larger terms."""
    rng = np.random.default_rng(5)
    for E, K, tau in ((64, 8, 4.0), (256, 8, 2.0), (8, 1, 1.0), (60, 60, 1.0)):
        xt, x = _logits(rng, 500, E, torch.float32)
        for near in (0.0, 1e-3, 1e-2):
            idx, logit, lse = _teacher(rng, x, K, K < E, tau, near)
            loss = rs.route_distill(xt, _dev(idx.astype(np.int32)), _dev(logit), None if lse is None else _dev(lse), temperature=tau).double().cpu().numpy()
            want = R.distill(x, idx, logit.astype(float), None if lse is None else lse.astype(float), tau)
            # errors of d of 200 u times |p - q| (about near / tau), and their square
            assert np.abs(loss - want).max() < tau * tau * (200 * U * near / tau + (200 * U) ** 2 + (0 if K < E else 4 * U * U)) + 1e-12


@pytest.mark.parametrize("far", [5.0, 12.0, 16.0, 40.0, 80.0, 120.0])
def test_a_student_sure_of_the_list_and_a_teacher_that_is_not(far):
    """The rest of the student's probability down to nothing, against a rest of the teacher's: the logarithm of their ratio, not of a difference."""
    rng = np.random.default_rng(6)
    T, E, K = 64, 32, 4
    x = rng.normal(size=(T, E)).astype(np.float32)
    x[:, :K] += np.float32(far)
    idx = np.tile(np.arange(K), (T, 1))
    logit = rng.normal(size=(T, K)).astype(np.float32)
    lse = (np.log(np.exp(logit.astype(float)).sum(axis=1)) + 0.4).astype(np.float32)
    loss = rs.route_distill(_dev(x), _dev(idx.astype(np.int32)), _dev(logit), _dev(lse))
    o = R.distill_terms(x.astype(float), idx, logit.astype(float), lse.astype(float))
    assert (o["rest_q"] > 0.3).all()
    want = R.distill(x.astype(float), idx, logit.astype(float), lse.astype(float))
    none = o["rest_p"] < 2.0 ** -126                        # the rest is left out where fp32 has nothing to hold against it
    if none.any():
        o["rest_q"] = np.where(none, 0.0, o["rest_q"])
        log_p = np.take_along_axis(o["z"], o["at"], 1) - o["lse"][:, None]
        want = np.where(none, (o["q"] * (o["u"] - o["log_mass"][:, None] - log_p)).sum(axis=1), want)
    near_border = np.abs(np.log2(np.maximum(o["rest_p"], 1e-300)) + 126) < 1e-3
    assert not near_border.any()
    # terms of up to 0.4 far and their relative errors of (10 Z + 2.5 far + 70) u
    _near(loss, want, (1 + np.abs(want)) * (10 * np.abs(x).max() + 2.5 * far + 100) * U, "loss")
    g = rs.route_distill_backward(_dev(x), _dev(idx.astype(np.int32)), _dev(logit), torch.ones(T, device=DEV), _dev(lse))
    wd, size = R.distill_backward(x.astype(float), idx, logit.astype(float), np.ones(T), lse.astype(float))
    assert bool(g.isfinite().all())
    some = ~none
    # outside the list q_r p_e / p_r: p_e and p_r each off by (10 Z + 2.5 far + 70) u of themselves, and what lies below fp32's normal range by all of it
    tol = np.abs(size) * 3 * (10 * np.abs(x).max() + 2.5 * far + 100) * U + 2 * 2.0 ** -126 * (1 + 1 / np.maximum(o["rest_p"], 2.0 ** -126))[:, None]
    _near(g[_dev(some)], wd[some], tol[some], "gradient")


def test_no_rows_and_no_groups():
    x = torch.empty((0, 8), device=DEV)
    idx = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    logp, lse, entropy, ai, al = rs.route_logprobs(x, idx, alternatives=2)
    assert logp.shape == (0, 2) and lse.shape == (0,) and ai.shape == (0, 2)
    assert rs.route_logprobs_backward(x, idx, logp, lse).shape == (0, 8)
    counts, tokens, sums, loss = rs.route_balance(x, idx, groups=3)
    assert not counts.any() and not tokens.any() and not sums.any() and not loss.any() and counts.shape == (3, 8)
    assert rs.route_balance_backward(x, 2, counts, tokens, loss).shape == (0, 8)
    assert rs.route_distill(x, idx, logp).shape == (0,) and rs.route_distill_backward(x, idx, logp, lse).shape == (0, 8)
    y = torch.randn((5, 8), device=DEV)
    picks = torch.zeros((5, 2), dtype=torch.int32, device=DEV)
    counts, tokens, sums, loss = rs.route_balance(y, picks, group_off=torch.zeros(1, dtype=torch.int64, device=DEV))
    assert counts.shape == (0, 8) and loss.shape == (0,)
    assert not rs.route_balance_backward(y, 2, counts, tokens, loss, group_off=torch.zeros(1, dtype=torch.int64, device=DEV)).any()
    nothing = rs.route_balance(y, picks, groups=1, row_mask=torch.zeros(5, dtype=torch.bool, device=DEV))
    assert not any(v.any() for v in nothing)


def test_offsets_outside_the_rows_are_clamped():
    rng = np.random.default_rng(8)
    xt, x = _logits(rng, 300, 16, torch.float32)
    it, idx = _picks(rng, 300, 16, 2)
    off = torch.tensor([-(1 << 40), 100, 250, 1 << 40], device=DEV)
    counts, tokens, sums, loss = rs.route_balance(xt, it, group_off=off)
    wc, wn, ws, wl = R.balance(x, idx, [(0, 100), (100, 250), (250, 300)], 1.0)
    np.testing.assert_array_equal(counts.cpu().numpy(), wc)
    _near(loss, wl, 1e-4, "loss")


def test_many_short_groups_and_one_long():
    rng = np.random.default_rng(9)
    T, E, k = 40_000, 60, 4
    xt, x = _logits(rng, T, E, torch.float32)
    it, idx = _picks(rng, T, E, k)
    lengths = rng.integers(0, 4, size=5000)
    cuts = np.concatenate([[0], np.cumsum(lengths)])
    cuts = np.concatenate([cuts, [T - 3, T - 3, T]])        # then one group of most rows, an empty one, three rows
    edges = list(zip(cuts[:-1], cuts[1:]))
    counts, tokens, sums, loss = rs.route_balance(xt, it, group_off=_dev(cuts), coef=1.0)
    wc, wn, ws, wl = R.balance(x, idx, edges, 1.0)
    np.testing.assert_array_equal(counts.cpu().numpy(), wc)
    np.testing.assert_array_equal(tokens.cpu().numpy(), wn)
    worst = _delta(x, 1.0).max() + 2.5 * U
    rows = wn[:, None] * np.ones((1, E))
    _near(sums, ws, ws * (worst + rows * U) + rows * U, "prob_sum")
    d = rng.normal(size=len(edges)).astype(np.float32)
    got = rs.route_balance_backward(xt, k, counts, tokens, _dev(d), group_off=_dev(cuts))
    want, size = R.balance_backward(x, k, edges, 1.0, wc, wn, d.astype(float))
    _gradient_near(got, want, size, x, 1.0, torch.float32, 8, 3 * _delta(x, 1.0), "gradient")


def test_rows_beyond_2_31_elements():
    """Row offsets of more than 31 bits: few rows, far apart."""
    rng = np.random.default_rng(10)
    T, E, ld = 2100, 16, 1 << 20
    memory = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV)
    xt = memory.view(T, ld)[:, :E]
    xt.copy_(_dev(rng.normal(size=(T, E))).to(torch.bfloat16))
    x = xt.double().cpu().numpy()
    it, idx = _picks(rng, T, E, 2)
    logp = rs.route_logprobs(xt, it)[0]
    _near(logp, R.logprobs(x, idx)[0], 200 * U, "logp")
    g = rng.normal(size=(T, 2)).astype(np.float32)
    grad = memory.view(T, ld)[:, E:2 * E]                   # between the rows of the logits: the same memory, other places
    rs.route_logprobs_backward(xt, it, _dev(g), out=grad)
    want, size = R.logprobs_backward(x, idx, g.astype(float), np.zeros(T), np.zeros(T))
    _gradient_near(grad, want, size, x, 1.0, torch.bfloat16, 2, 3 * _delta(x, 1.0), "gradient")
    assert bool((xt.double().cpu() == torch.from_numpy(x)).all())
    wide = memory.view(-1)[:(1 << 31) + 512].view(-1, 512)  # and many rows
    wide.normal_()
    T = wide.shape[0]
    some = torch.zeros((T, 1), dtype=torch.int32, device=DEV)
    lse = rs.route_logprobs(wide, some)[1]
    tail = wide[-1000:].double().cpu().numpy()
    _near(lse[-1000:], R.softmax(tail)[3], 200 * U, "lse of the last rows")


# ------------------------------------------------------------------------------------------------ how it is called
def _everything(x, it, teacher, mask, n=4):
    """All operators once; a list of tensors."""
    T, k = it.shape
    logp, lse, entropy, ai, al = rs.route_logprobs(x, it, alternatives=4, row_mask=mask)
    counts, tokens, sums, loss = rs.route_balance(x, it, groups=n, coef=0.01, row_mask=mask)
    d = rs.route_logprobs_backward(x, it, torch.ones_like(logp), lse * 1e-3, torch.full_like(entropy, 0.1), row_mask=mask)
    rs.route_balance_backward(x, k, counts, tokens, torch.ones_like(loss), coef=0.01, row_mask=mask, accumulate=True, out=d)
    kl = rs.route_distill(x, teacher[0], teacher[1], teacher[2], row_mask=mask)
    rs.route_distill_backward(x, *teacher[:2], torch.full_like(kl, 0.5), teacher[2], row_mask=mask, accumulate=True, out=d)
    return [logp, lse, entropy, ai, al, counts, tokens, sums, loss, kl, d]


def _inputs(seed, T=4096, E=64, k=6, dtype=torch.float32):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((T, E), device=DEV, generator=gen).to(dtype)
    it = torch.randint(0, E, (T, k), device=DEV, generator=gen).to(torch.int32)
    it[5] = 7                                               # one expert in every slot: an order of additions that has to be kept
    t = torch.randn((T, E), device=DEV, generator=gen).topk(k)
    ti = t.indices.to(torch.int32)
    ti[6] = 9
    mask = (torch.rand(T, device=DEV, generator=gen) > 0.1).to(torch.uint8)
    return x, it, (ti, t.values.contiguous(), torch.full((T,), 4.0, device=DEV)), mask


@pytest.mark.parametrize("E,dtype", [(8, "fp32"), (61, "fp32"), (64, "bf16"), (256, "fp32"), (1000, "fp16")])
def test_equal_inputs_give_equal_bits(E, dtype):
    args = _inputs(1, 4096, E, 6, TYPES[dtype])
    first = _everything(*args)
    for _ in range(3):
        for a, b in zip(first, _everything(*args)):
            assert torch.equal(a, b)


def test_rows_do_not_depend_on_their_place():
    """A row's results are the same bits alone and among others."""
    for E in (8, 61, 64, 256, 512):
        x, it, teacher, _ = _inputs(2, 300, E, 4)
        whole = rs.route_logprobs(x, it, alternatives=4)
        kl = rs.route_distill(x, *teacher)
        d = rs.route_distill_backward(x, *teacher[:2], torch.ones(300, device=DEV), teacher[2])
        for r in (0, 5, 6, 131, 299):
            alone = rs.route_logprobs(x[r:r + 1], it[r:r + 1], alternatives=4)
            for a, b in zip(whole, alone):
                assert torch.equal(a[r:r + 1], b)
            part = [v[r:r + 1] for v in teacher]
            assert torch.equal(kl[r:r + 1], rs.route_distill(x[r:r + 1], *part))
            assert torch.equal(d[r:r + 1], rs.route_distill_backward(x[r:r + 1], *part[:2], torch.ones(1, device=DEV), part[2]))


def test_another_stream():
    args = _inputs(3)
    want = _everything(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _everything(*args)
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,E,n", [(4096, 64, 4), (70_000, 256, 1), (1000, 8, 8)])
def test_captured_and_replayed(T, E, n):
    """Two graphs with workspaces of their own, replayed in turn with eager work between them, on new inputs."""
    x, it, teacher, mask = _inputs(4, T, E)
    _everything(x, it, teacher, mask, n)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _everything(x, it, teacher, mask, n)
        graphs.append((g, out))
    for seed in (5, 6, 7):
        y, jt, other, mask2 = _inputs(seed, T, E)
        x.copy_(y)
        it.copy_(jt)
        for a, b in zip(teacher, other):
            a.copy_(b)
        mask.copy_(mask2)
        want = _everything(x, it, teacher, mask, n)
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(want, out):
                assert torch.equal(a, b)


def test_a_training_step_of_a_router():
    """The operators as they are used together: the picks of stage 1, gate weights, z-loss, balance over sequences, one gradient; then a forecaster
    trained on the router's own lists, and the forecast routed."""
    rng = np.random.default_rng(11)
    T, E, k, K = 2000, 64, 6, 8
    xt, x = _logits(rng, T, E, torch.float32)
    it = rs.route_topk(xt.contiguous(), k)
    idx = it.cpu().numpy()
    cuts = np.array([0, 300, 301, 1500, 2000])
    edges = list(zip(cuts[:-1], cuts[1:]))
    logp, lse, entropy, ai, al = rs.route_logprobs(xt, it, alternatives=K)
    np.testing.assert_array_equal(ai[:, :k].cpu().numpy(), idx)                     # the most likely experts are stage 1's picks
    assert torch.equal(al[:, :k], logp)
    counts, tokens, sums, loss = rs.route_balance(xt, it, group_off=_dev(cuts), coef=0.01)
    weights = logp.exp()
    d_weights = _dev(rng.normal(size=(T, k)).astype(np.float32))
    d = rs.route_logprobs_backward(xt, it, d_weights * weights, 2e-3 * lse)          # of the weights, and of 1e-3 lse^2
    rs.route_balance_backward(xt, k, counts, tokens, torch.ones(4, device=DEV), group_off=_dev(cuts), coef=0.01, accumulate=True, out=d)
    w64 = (d_weights * weights).double().cpu().numpy()
    a, sa = R.logprobs_backward(x, idx, w64, (2e-3 * lse).double().cpu().numpy(), np.zeros(T))
    c64 = R.balance(x, idx, edges, 0.01)
    b, sb = R.balance_backward(x, k, edges, 0.01, c64[0], c64[1], np.ones(4))
    _gradient_near(d, a + b, sa + sb, x, 1.0, torch.float32, k, 4 * _delta(x, 1.0), "summed gradient")

    student, s64 = _logits(rng, T, E, torch.bfloat16)
    none = torch.zeros(T, device=DEV)                                                # log probabilities: their log-sum-exp is 0
    kl = rs.route_distill(student, ai, al, none)
    want = R.distill(s64, ai.cpu().numpy(), al.double().cpu().numpy(), np.zeros(T))
    _near(kl, want, 1e-4 * (1 + want), "divergence")
    step = rs.route_distill_backward(student, ai, al, none + 1.0, none)
    nearer = rs.route_distill((student.float() - 0.5 * step.float()).to(torch.bfloat16), ai, al, none)
    assert float(nearer.mean()) < float(kl.mean())                                   # a step against the gradient
    M, N = 4, 4
    table = torch.arange(E, dtype=torch.int32, device=DEV).remainder(M * N).view(E, 1).contiguous()
    topo = rs.Topo(M, N, 65536)
    D1 = rs.route_traffic(student.float().contiguous(), k, 1, T // (M * N), table, 4096, topo)[1]
    assert int(D1.sum()) == T * k * 4096


def test_refusals_on_the_device():
    x, it, teacher, mask = _inputs(12, 64, 16, 4)
    two = torch.zeros(64, device=DEV)
    for bad in (lambda: rs.route_logprobs(x.double(), it), lambda: rs.route_logprobs(x.t(), it), lambda: rs.route_logprobs(x[0], it),
                lambda: rs.route_logprobs(x[:1].expand(64, 16), it), lambda: rs.route_logprobs(x, it.long()), lambda: rs.route_logprobs(x, it[:5]),
                lambda: rs.route_logprobs(x, it[0]), lambda: rs.route_logprobs(x, it.cpu()), lambda: rs.route_logprobs(x, it, row_mask=mask[:5]),
                lambda: rs.route_logprobs_backward(x, it, two[:1].expand(64, 4)),            # a broadcast gradient is laid out first
                lambda: rs.route_logprobs_backward(x, it, accumulate=True),
                lambda: rs.route_logprobs_backward(x, it, out=x.to(torch.bfloat16)), lambda: rs.route_balance(x, it, group_off=mask),
                lambda: rs.route_balance(x, it, group_off=torch.empty(0, dtype=torch.int64, device=DEV)),
                lambda: rs.route_distill(x, teacher[0], teacher[1][:, :2]), lambda: rs.route_distill(x, teacher[0], teacher[1], two[:3])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: rs.route_logprobs(x, it, alternatives=17), lambda: rs.route_logprobs(x, it, temperature=0.0), lambda: rs.route_balance(x, it, groups=3),
                lambda: rs.route_logprobs_backward(x, it, out=x), lambda: rs.route_logprobs(x, it, out=(None, None, None, None, None)),
                lambda: rs.route_balance(x, it, ws=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises(rs.RailschedError):
            bad()


# ------------------------------------------------------------------------------------------------ the ways through the kernels
@pytest.mark.parametrize("E", [8, 12, 32, 36, 40, 64, 68, 100, 128, 132, 240, 256, 260, 511, 512, 516, 1000, 1024])
@pytest.mark.parametrize("kind", ["few values", "neighbours", "bf16", "mostly out"])
def test_alternatives_in_stage_1s_order(E, kind):
    """Ties, values a step apart and experts that are out, in every way of finding the largest: the order is that of a stable sort."""
    rng = np.random.default_rng(E)
    T = 260
    if kind == "few values":
        x = rng.integers(-2, 3, size=(T, E)).astype(np.float32)
        x[x == 0] *= -1                                     # -0 and +0 are equal
    elif kind == "neighbours":
        x = (np.float32(1.0) + rng.integers(0, 6, size=(T, E)) * np.float32(2.0 ** -23)).astype(np.float32)
        x *= np.where(rng.random((T, 1)) < 0.5, np.float32(-1), np.float32(1))
    elif kind == "bf16":
        x = rng.normal(size=(T, E)).astype(np.float32)
    else:
        x = np.where(rng.random((T, E)) < 0.97, -np.inf, rng.normal(size=(T, E))).astype(np.float32)
    xt = _dev(x)
    if kind == "bf16":
        xt = xt.to(torch.bfloat16)
        x = xt.float().cpu().numpy()
    order = np.argsort(-x, axis=1, kind="stable")
    for m in sorted({1, min(E, 4), min(E, 8), min(E, 9), min(E, 16), min(E, 17), min(E, 64)}):
        ai, al = rs.route_logprobs(xt, alternatives=m)[3:]
        want = np.where(np.take_along_axis(x, order[:, :m], 1) == -np.inf, -1, order[:, :m])
        np.testing.assert_array_equal(ai.cpu().numpy(), want, err_msg=f"{m} alternatives")
        wa = R.logprobs(x.astype(float), np.zeros((T, 0), int), m)[4]
        _near(al, wa, (10 * np.abs(x[np.isfinite(x)]).max() + 80 + 8) * U, f"{m} alternatives")


def test_a_grid_of_two_dimensions():
    """More workgroups than one dimension of a grid takes here: 2^28 rows of two logits."""
    T = (1 << 28) + 100
    x = torch.zeros((T, 2), dtype=torch.bfloat16, device=DEV)
    x[-50:, 0] = 1.0
    x[:50, 1] = 2.0
    lse = rs.route_logprobs(x)[1]
    grad = rs.route_logprobs_backward(x, d_lse=torch.ones(T, device=DEV))
    spread = rs.route_balance_backward(x, 1, torch.tensor([[3, 1]], device=DEV), torch.tensor([4], device=DEV), torch.ones(1, device=DEV))
    for part in (slice(0, 1000), slice((1 << 27) - 500, (1 << 27) + 500), slice(T - 1000, T)):
        at = x[part].double().cpu().numpy()
        _near(lse[part], R.softmax(at)[3], 200 * U, "lse")
        want, size = R.logprobs_backward(at, np.zeros((1000, 0), int), np.zeros((1000, 0)), np.ones(1000), np.zeros(1000))
        _gradient_near(grad[part], want, size, at, 1.0, torch.bfloat16, 0, 3 * _delta(at, 1.0), "gradient of lse")
        want, size = R.balance_backward(at, 1, [(0, 1000)], 1.0, np.array([[3, 1]]), np.array([4]), np.ones(1))
        _gradient_near(spread[part], want, size, at, 1.0, torch.bfloat16, 8, 3 * _delta(at, 1.0), "gradient of the balance loss")
    counts, tokens, sums, loss = rs.route_balance(x, torch.zeros((T, 1), dtype=torch.int32, device=DEV))
    assert int(tokens) == T and counts.tolist() == [[T, 0]] and abs(float(sums.double().sum()) / T - 1) < 1e-5


@pytest.mark.parametrize("groups", [1, 3, 16, 512, 4096])
@pytest.mark.parametrize("E,dtype", [(8, "fp32"), (60, "bf16"), (61, "fp32"), (256, "fp32"), (512, "fp16"), (1024, "bf16")])
def test_balance_of_equal_groups(groups, E, dtype):
    """Groups in a workgroup of their own, in slices, in slices of the larger workgroups, with one tile of columns and several."""
    rng = np.random.default_rng(groups + E)
    dtype = TYPES[dtype]
    for each in sorted({1, 37, (1 << 16) // groups // max(1, E // 64) + 1}):
        T, k = groups * each, 2
        if T * E > 1 << 23:
            continue
        xt, x = _logits(rng, T, E, dtype)
        it, idx = _picks(rng, T, E, k)
        mt, mask = _mask(rng, T)
        counts, tokens, sums, loss = rs.route_balance(xt, it, groups=groups, coef=1.0, row_mask=mt)
        wc, wn, ws, wl = R.balance(x, idx, [(g * each, (g + 1) * each) for g in range(groups)], 1.0, mask)
        np.testing.assert_array_equal(counts.cpu().numpy(), wc)
        np.testing.assert_array_equal(tokens.cpu().numpy(), wn)
        worst = _delta(x, 1.0).max() + each * U
        _near(sums, ws, worst * ws + 2 * each * U, "prob_sum")
        share = E / (k * np.maximum(wn, 1.0) ** 2) * wc.sum(axis=1)
        _near(loss, wl, wl * (worst + 2 * U) + share * 2 * each * U, "loss")


def test_a_dirty_workspace_and_one_for_two_calls():
    rng = np.random.default_rng(13)
    for T, E, groups in ((5000, 64, 5), (70_000, 256, 1), (40, 8, 4)):
        xt, x = _logits(rng, T, E, torch.float32)
        it, _ = _picks(rng, T, E, 4)
        yt, _ = _logits(rng, T, E, torch.float32)
        want = [v.clone() for v in rs.route_balance(xt, it, groups=groups)], [v.clone() for v in rs.route_balance(yt, it, groups=groups)]
        ws = torch.full((rs.route_balance_workspace_bytes(T, groups, E),), 0xFF, dtype=torch.uint8, device=DEV)
        got = rs.route_balance(xt, it, groups=groups, ws=ws), rs.route_balance(yt, it, groups=groups, ws=ws)     # in order on one stream
        for a, b in zip(want, got):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_a_teacher_whose_mass_is_off():
    """A log-sum-exp that is too small (the list alone exceeds it: no rest) or too large (a rest that is not the teacher's) is taken as it is given."""
    rng = np.random.default_rng(14)
    for E, K in ((64, 8), (61, 61), (256, 16)):
        xt, x = _logits(rng, 300, E, torch.float32)
        idx, logit, lse = _teacher(rng, x, K, True, 1.0)
        for shift in (-3.0, -0.7, 0.7, 3.0):
            given = (lse + np.float32(shift)).astype(np.float32)
            args = _dev(idx.astype(np.int32)), _dev(logit)
            loss = rs.route_distill(xt, *args, _dev(given))
            want = R.distill(x, idx, logit.astype(float), given.astype(float))
            # q up to e^3: its error, that of p and of the logarithms, each of (10 Z + 70) u, times what is added up
            size = 1 + np.exp(-shift) * (10 + np.abs(shift))
            _near(loss, want, 4 * size * (10 * max(np.abs(x).max(), np.abs(given).max()) + 110) * U, f"loss of {E}, {shift}")
            g = rs.route_distill_backward(xt, *args, torch.ones(300, device=DEV), _dev(given))
            wd, mag = R.distill_backward(x, idx, logit.astype(float), np.ones(300), given.astype(float))
            o = R.distill_terms(x, idx, logit.astype(float), given.astype(float))
            mag = mag + o["p"] * np.where(o["rest_q"] > 0, (o["mass"] + 1) / np.maximum(o["rest_p"], 1e-300), 0.0)[:, None]
            _near(g, wd, 4 * mag * (10 * max(np.abs(x).max(), np.abs(given).max()) + 110) * U + 2.0 ** -126, f"gradient of {E}, {shift}")


def test_two_streams_at_once():
    """Calls that run at the same time on buffers of their own do not reach each other."""
    a, b = _inputs(15, 60_000, 256), _inputs(16, 60_000, 60)
    want = _everything(*a), _everything(*b)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [[], []]
    for _ in range(4):
        for i, args in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(_everything(*args))
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        for r in runs:
            assert all(torch.equal(u, v) for u, v in zip(w, r))


@pytest.mark.parametrize("groups", [2, 20, 150, 1500])
@pytest.mark.parametrize("E,dtype", [(2, "fp16"), (7, "fp32"), (33, "bf16"), (64, "fp32"), (100, "fp32"), (256, "bf16"), (300, "fp32"), (891, "fp16")])
def test_balance_of_ragged_groups(groups, E, dtype):
    """Groups cut into few and many records, whose columns are joined in one tile or several."""
    rng = np.random.default_rng(groups * 3 + E)
    dtype = TYPES[dtype]
    T, k = min((1 << 23) // E, 400_000) - 5, 2
    xt, x = _logits(rng, T, E, dtype)
    it, idx = _picks(rng, T, E, k)
    mt, mask = _mask(rng, T)
    cuts = np.sort(rng.integers(0, T + 1, size=groups + 1))
    counts, tokens, sums, loss = rs.route_balance(xt, it, group_off=_dev(cuts), coef=1.0, row_mask=mt)
    wc, wn, ws, wl = R.balance(x, idx, list(zip(cuts[:-1], cuts[1:])), 1.0, mask)
    np.testing.assert_array_equal(counts.cpu().numpy(), wc)
    np.testing.assert_array_equal(tokens.cpu().numpy(), wn)
    # as for the groups above: a group's sum is off by its terms, and by as many additions in fp32 as it has rows at most
    worst = _delta(x, 1.0).max() + wn[:, None] * U
    _near(sums, ws, worst * ws + 2 * wn[:, None] * U, "prob_sum")
    share = E / (k * np.maximum(wn, 1.0) ** 2) * wc.sum(axis=1)
    _near(loss, wl, wl * (worst[:, 0] + 2 * U) + share * 2 * wn * U, "loss")


@pytest.mark.parametrize("E", [5, 6, 7, 33, 45, 61, 67, 130, 251, 510, 1021])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_rows_that_end_with_a_part_of_a_four(E, dtype):
    """The same bits as with experts that are out up to the next multiple of four, wherever the rows lie, and nothing beside the rows is written."""
    rng = np.random.default_rng(E)
    dtype, T, k, W = TYPES[dtype], 300, 2, -(-E // 4) * 4
    padded = torch.full((T, W), -float("inf"), dtype=dtype, device=DEV)
    padded[:, :E], _ = _logits(rng, T, E, dtype, out=0.1)
    it, _ = _picks(rng, T, E, k, strange=False)             # an index of E is no expert of one side, and of the other one that is out
    teacher = _logits(rng, T, 4, torch.float32)[0], torch.full((T,), 3.0, device=DEV)
    ti = _dev(rng.integers(0, E, size=(T, 4)).astype(np.int32))
    g = _dev(rng.normal(size=(T, k)).astype(np.float32))

    def everything(x, place):
        outs = [v for m in (0, 1, min(E, 8), min(E, 16)) for v in rs.route_logprobs(x, it, alternatives=m) if v is not None]
        counts, tokens, sums, loss = rs.route_balance(x, it)
        outs += [counts[:, :E], tokens, sums[:, :E], rs.route_distill(x, ti, teacher[0], teacher[1])]
        grads = []
        for add in (False, True):
            grads.append(rs.route_logprobs_backward(x, it, g, g[:, 0].contiguous(), g[:, 1].contiguous(), accumulate=add, out=place).clone())
            grads.append(rs.route_balance_backward(x, k, counts, tokens, torch.ones(1, device=DEV), accumulate=add, out=place).clone())
            grads.append(rs.route_distill_backward(x, ti, teacher[0], g[:, 0].contiguous(), teacher[1], accumulate=add, out=place).clone())
        return outs, [v[:, :E] for v in grads]

    want, want_grads = everything(padded, torch.empty_like(padded))
    for shift in range(4):
        for ld in (E, E + 1, W):
            room = torch.full((T * ld + 8,), 5.0, dtype=dtype, device=DEV)
            x = room[shift:shift + T * ld].view(T, ld)[:, :E]
            x.copy_(padded[:, :E])
            to = torch.full((T * ld + 8,), 7.0, dtype=dtype, device=DEV)
            place = to[3 - shift:3 - shift + T * ld].view(T, ld)[:, :E]
            got, grads = everything(x, place)
            what = f"{shift} values off, {ld} apart"
            if shift == 0 and ld == E:                      # a balance loss counts the experts, and its gradient is in these
                for i in (1, 4, 5):
                    want_grads[i] = grads[i]
            for a, b in zip(want, got):
                assert torch.equal(a, b), what
            for a, b in zip(want_grads, grads):
                assert torch.equal(a, b), what
            place.fill_(7.0)
            assert bool((to == 7.0).all()), what


@pytest.mark.parametrize("cuts", [[0, 0], [100, 100, 100], [7, 400, 993], [0, 500, 1000], [1000, 1000], [640, 1000], [0, 3]])
@pytest.mark.parametrize("E,dtype", [(8, "fp32"), (61, "bf16"), (256, "fp32")])
def test_rows_of_no_group_have_no_gradient(cuts, E, dtype):
    """Without `out` the rows before the first group and behind the last one are 0, whatever they hold; the others are what they are with it."""
    rng = np.random.default_rng(E)
    T, k = 1000, 2
    xt, _ = _logits(rng, T, E, TYPES[dtype])
    it, _ = _picks(rng, T, E, k)
    xt[:cuts[0]] = float("nan")
    xt[cuts[-1]:] = float("inf")
    off = torch.tensor(cuts, device=DEV)
    counts, tokens, _, loss = rs.route_balance(xt, it, group_off=off)
    want = torch.zeros_like(xt)
    rs.route_balance_backward(xt, k, counts, tokens, torch.ones_like(loss), group_off=off, out=want)
    for _ in range(2):
        dirty = torch.full_like(xt, float("nan"))           # what the allocator hands out next
        del dirty
        got = rs.route_balance_backward(xt, k, counts, tokens, torch.ones_like(loss), group_off=off)
        assert torch.equal(got, want)
    assert not bool(want[:cuts[0]].any()) and not bool(want[cuts[-1]:].any()) and bool(want.isfinite().all())


def test_no_group_at_all_has_no_gradient():
    x = torch.randn((50, 8), device=DEV)
    none = torch.zeros((0, 8), dtype=torch.int64, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, device=DEV)
    assert not bool(rs.route_balance_backward(x, 2, *none, group_off=torch.zeros(1, dtype=torch.int64, device=DEV)).any())
