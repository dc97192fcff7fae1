"""The operators on a router's logits where their arguments are at the edge of what the header allows.  Tolerances as derived in test_gpu_router.py."""
import numpy as np
import pytest
import torch

from oracle import router as R
from test_gpu_router import DEV, TYPES, U, _delta, _dev, _gradient_near, _logits, _near, _picks, _teacher

pytestmark = pytest.mark.gpu

rs = pytest.importorskip("paper_2510_19262_amd")


@pytest.mark.parametrize("E", [3, 8, 11, 27, 61, 64, 256, 1000])
@pytest.mark.parametrize("size", [1.0, 1e9, -1e30, 1e37])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_entropy_gradient_of_any_size_where_experts_are_out(E, size, dtype):
    """p (log p + entropy) is 0 for an expert that is out and small for one that nearly is, whatever d_entropy it is multiplied with."""
    rng = np.random.default_rng(E)
    T, dtype = 70, TYPES[dtype]
    xt, x = _logits(rng, T, E, dtype, out=0.4)
    for t in (xt, x):
        t[1, 0], t[1, 1], t[1, 2] = 1.0, -79.0, -float("inf")      # p of 2^-115: in fp32's normal range
        t[2, 0], t[2, 1:] = 3.0, -float("inf")                      # one expert left: the entropy does not move
    mt = torch.ones(T, dtype=torch.uint8, device=DEV)
    mt[5] = 0
    xt[5] = float("nan")
    mask = mt.cpu().numpy()
    x[5] = 0.0
    idx = np.zeros((T, 1), int)
    it = _dev(idx.astype(np.int32))
    d_h = (rng.uniform(0.5, 1.0, size=T) * size).astype(np.float32)
    g = rng.normal(size=(T, 1)).astype(np.float32)
    for with_logp in (False, True):
        a = g if with_logp else np.zeros_like(g)
        got = rs.route_logprobs_backward(xt, it if with_logp else None, _dev(g) if with_logp else None, None, _dev(d_h), row_mask=mt)
        want, mag = R.logprobs_backward(x, idx, a.astype(float), np.zeros(T), d_h.astype(float), 1.0, mask)
        out = _dev(x == -np.inf)
        out[:, 0] &= not with_logp                                  # a pick that is out has its slot's gradient
        assert not bool(got[out].any())
        _gradient_near(got, want, mag, x, 1.0, dtype, 1, 3 * _delta(x, 1.0), "gradient")


@pytest.mark.parametrize("rows,E", [(1, 1), (5, 8), (300, 11), (70, 61), (4000, 64), (33, 1024)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradient_without_a_group_through_the_c_entry(rows, E, dtype):
    """accumulate = 2 sets every row to 0 where there is no group, whatever the rows, the mask and the memory hold; 0 and 1 leave them."""
    from paper_2510_19262_amd import binding
    code, dtype = binding.DTYPES[TYPES[dtype]], TYPES[dtype]
    x = torch.full((rows, E), float("nan"), dtype=dtype, device=DEV)
    mt = torch.zeros(rows, dtype=torch.uint8, device=DEV)
    for first in (-3, 0, rows // 2, rows, 1 << 40):
        off = torch.tensor([first], device=DEV)
        for mask in (None, mt.data_ptr()):
            for how in (2, 0, 1):
                place = torch.full((rows + 1, E + 3), 7.0, dtype=dtype, device=DEV)
                place[:rows, :E] = float("nan")
                rc = rs.load().railsched_route_balance_backward(x.data_ptr(), code, rows, E, E, mask, 1, off.data_ptr(), 0, 1.0, None, None, None, how,
                                                                place.data_ptr(), E + 3, torch.cuda.current_stream().cuda_stream)
                assert rc == 0
                d = place[:rows, :E]
                assert bool((d == 0).all()) if how == 2 else bool(d.isnan().all())
                assert bool((place[:, E:] == 7.0).all()) and bool((place[rows] == 7.0).all())


def test_gradient_without_a_group_is_checked_as_any_other():
    x = torch.randn((50, 8), device=DEV)
    none = torch.zeros((0, 8), dtype=torch.int64, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV), torch.zeros(0, device=DEV)
    off = torch.zeros(1, dtype=torch.int64, device=DEV)
    dirty = torch.full_like(x, float("nan"))                # what the allocator hands out next
    del dirty
    assert torch.equal(rs.route_balance_backward(x, 2, *none, group_off=off), torch.zeros_like(x))
    for k in (0, 9):
        with pytest.raises(rs.RailschedError):
            rs.route_balance_backward(x, k, *none, group_off=off)
    with pytest.raises(ValueError):
        rs.route_balance_backward(x, 2, none[0], none[1].int(), none[2], group_off=off)


@pytest.mark.parametrize("groups,E,rows", [((1 << 22) - 1, 257, 3000), (1 << 22, 257, 3000), (1 << 22, 700, 0), ((1 << 22) + 5, 513, 999), (1 << 23, 260, 5000), (1 << 23, 8, 5000)])
def test_as_many_groups_as_there_may_be(groups, E, rows):
    """Most of them empty; up to 2^23, whatever the number of experts."""
    rng = np.random.default_rng(groups % 1000 + E)
    xt, x = _logits(rng, rows, E, torch.float32)
    k = 2
    idx = rng.integers(0, E, size=(rows, k))
    cuts = np.sort(rng.integers(0, rows + 1, size=groups + 1))
    cuts[0], cuts[-1] = 0, rows
    off = _dev(cuts)
    counts, tokens, sums, loss = rs.route_balance(xt, _dev(idx.astype(np.int32)), group_off=off, coef=1.0)
    n = np.diff(cuts)
    assert torch.equal(tokens, _dev(n))
    some = np.flatnonzero(n)
    edges = [(int(cuts[g]), int(cuts[g + 1])) for g in some]
    wc, wn, ws, wl = R.balance(x, idx, edges, 1.0)
    at = _dev(some)
    assert torch.equal(counts[at], _dev(wc)) and int(counts.sum()) == rows * k
    most = max(int(n.max()), 1) if rows else 1
    worst = (_delta(x, 1.0).max() if rows else 0.0) + most * U
    _near(sums[at], ws, worst * ws + 2 * most * U, "prob_sum")
    share = E / (k * np.maximum(wn, 1.0) ** 2) * wc.sum(axis=1)
    _near(loss[at], wl, wl * (worst + 2 * U) + share * 2 * most * U, "loss")
    empty = tokens == 0
    assert not bool(loss[empty].any()) and int((sums.amax(1) > 0).sum()) == len(some) and bool((sums.amin(1) >= 0).all())
    d = rs.route_balance_backward(xt, k, counts, tokens, torch.ones(groups, device=DEV), group_off=off)
    want, size = R.balance_backward(x, k, edges, 1.0, wc, wn, np.ones(len(some)))
    if rows:
        _gradient_near(d, want, size, x, 1.0, torch.float32, 8, 3 * _delta(x, 1.0), "gradient")
    del counts, sums, loss, tokens, d
    torch.cuda.empty_cache()


@pytest.mark.parametrize("E", [8, 32, 36, 61, 64, 100, 128, 250, 256, 400, 512, 1000, 1024])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_alternatives_of_rows_with_nan(E, dtype):
    """The numbers of such a row in their order, and no NaN, in every way of finding the largest and whatever rows are beside it."""
    rng = np.random.default_rng(E)
    T, inf, nan = 96, float("inf"), float("nan")
    xt, x = _logits(rng, T, E, TYPES[dtype])
    strange = np.arange(0, T, 5)                            # rows with NaN among rows without
    for i, r in enumerate(strange):
        at = rng.permutation(E)
        if i % 4 == 0:
            x[r, at[0]] = nan
        elif i % 4 == 1:                                    # few numbers left, -NaN and +NaN
            x[r] = -inf
            x[r, at[:3]] = [1.0, -2.0, 1.0]
            x[r, at[3:5]] = [nan, np.copysign(nan, -1.0)]
        elif i % 4 == 2:
            x[r, at[:2]] = [inf, nan]
        else:
            x[r] = nan
    xt.copy_(torch.from_numpy(x).to(DEV))
    ties = xt.clone()
    for r in range(T):
        if r not in strange:
            ties[r] = 1.0                                   # the rows beside them: all ties
    order = [[e for e in np.argsort(-np.where(np.isnan(row), -inf, row), kind="stable") if row[e] > -inf] for row in x]
    for m in sorted({1, min(E, 4), min(E, 8), min(E, 9), min(E, 16), min(E, 20)}):
        ai, al = rs.route_logprobs(xt, alternatives=m)[3:]
        for r in strange:
            want = (order[r] + [-1] * m)[:m]
            assert ai[r].tolist() == want, f"row {r}, {m} alternatives"
            assert all(np.isnan(v) if e >= 0 else v == -inf for e, v in zip(want, al[r].tolist()))
            alone = rs.route_logprobs(xt[r:r + 1], alternatives=m)[3:]
            assert torch.equal(alone[0][0], ai[r]) and torch.equal(alone[1][0].isnan(), al[r].isnan())
        beside, _ = rs.route_logprobs(ties, alternatives=m)[3:]
        assert torch.equal(beside[_dev(strange)], ai[_dev(strange)])
        for r in range(T):                                  # and they do not reach the others
            if r not in strange:
                assert ai[r].tolist() == order[r][:m]


@pytest.mark.parametrize("tau", [2.0 ** -8, 0.05, 32.0, 100.0, 256.0])
@pytest.mark.parametrize("E,K,tail", [(64, 8, False), (64, 64, False), (64, 8, True), (61, 20, True), (256, 16, True), (8, 8, False), (1000, 30, True)])
@pytest.mark.parametrize("near", [0.5, 2.0])
def test_distillation_at_the_ends_of_its_temperatures(tau, E, K, tail, near):
    """The bounds of test_gpu_router.test_distill hold up to the limits, where d = log p - log q is small (tau large) or its error is (tau small)."""
    rng = np.random.default_rng(E + K)
    T = 400
    xt, x = _logits(rng, T, E, torch.float32, scale=1.0)
    idx, logit, lse = _teacher(rng, x, K, tail, tau, near)
    args, lt, l64 = (_dev(idx.astype(np.int32)), _dev(logit)), None if lse is None else _dev(lse), None if lse is None else lse.astype(float)
    o = R.distill_terms(x, idx, logit.astype(float), l64, tau)
    if tail:                                                # rows whose rest fp32 leaves out have a test of their own
        fine = o["rest_p"] > 2.0 ** -100
        if not fine.any():
            pytest.skip("no row has a rest at this temperature")
    else:
        fine = np.ones(T, bool)
    want = R.distill(x, idx, logit.astype(float), l64, tau)
    loss = rs.route_distill(xt, *args, lt, temperature=tau)
    p = np.take_along_axis(o["p"], idx, 1)
    log_p = np.take_along_axis(o["z"], idx, 1) - o["lse"][:, None]
    d = np.abs(log_p - (o["u"] - o["log_mass"][:, None]))
    t = np.take_along_axis(x.max(axis=1, keepdims=True) - x, idx, 1) / tau
    delta = 2 * _delta(x, tau, np.abs(logit).max(axis=1) / tau, *([np.abs(lse)] if tail else [])) + 2.5 * U * t.max(axis=1)
    P = p.sum(axis=1)
    large = np.where(d > 0.25, p + o["q"] * (1 + d), 0.0).sum(axis=1)
    apart = np.abs(o["mass"] - P)
    rest = np.where(o["rest_q"] > 0, apart / np.maximum(o["rest_p"], 1e-300) * (o["mass"] + P), o["rest_p"] + (o["mass"] if tail else 0.0))
    # d's error in the second order too: delta^2, which is all there is where p is q
    tol = tau * tau * (delta * (np.abs(p - o["q"]).sum(axis=1) + large + rest) + delta * delta) + np.abs(want) * 64 * U + 2.0 ** -100
    _near(loss[_dev(fine)], want[fine], tol[fine], "loss")
    g = rng.normal(size=T).astype(np.float32)
    got = rs.route_distill_backward(xt, *args, _dev(g), lt, temperature=tau)
    wd, size = R.distill_backward(x, idx, logit.astype(float), g.astype(float), l64, tau)
    size = size + np.abs(tau * g)[:, None] * o["p"] * np.where(o["rest_q"] > 0, (o["mass"] + P) / np.maximum(o["rest_p"], 1e-300), 0.0)[:, None]
    _gradient_near(got[_dev(fine)], wd[fine], size[fine], x[fine], tau, torch.float32, K, 2 * delta[fine], "gradient")
    # and what the header says of either end: about 2^-11 of the gradient, or of tau d_loss, for differences of about 1; 2^-9 here, where they are 0.5 to several
    off = np.abs(got.double().cpu().numpy() - wd).sum(axis=1)[fine]
    assert (off <= 2.0 ** -9 * np.maximum(np.abs(wd).sum(axis=1), np.abs(tau * g))[fine]).all() if tau < 1 else (off <= 2.0 ** -9 * np.abs(wd).sum(axis=1)[fine]).all()


@pytest.mark.parametrize("by", [1 << 32, -(1 << 32), 1 << 40])
def test_numbers_that_32_bits_do_not_hold(by):
    """They are refused, not cut to their low bits."""
    x, it = torch.randn((4, 8), device=DEV), torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    counts, tokens, _, loss = rs.route_balance(x, it)
    for call in (lambda: rs.route_balance_backward(x, 2 + by, counts, tokens, loss), lambda: rs.route_logprobs(x, it, alternatives=2 + by),
                 lambda: rs.route_balance(x, it, groups=1 + by)):
        with pytest.raises(ValueError):
            call()


def test_logits_of_a_gate_that_autograd_trains():
    """What comes back is detached; the summed gradient goes on from the logits to the gate's weights."""
    rng = np.random.default_rng(21)
    T, H, E, k = 500, 16, 24, 4
    tokens, weight = rng.normal(size=(T, H)).astype(np.float32), rng.normal(size=(E, H)).astype(np.float32) * np.float32(0.25)
    w = _dev(weight).requires_grad_()
    logits = _dev(tokens) @ w.t()
    x = logits.detach().double().cpu().numpy()
    it = rs.route_topk(logits.detach(), k)
    idx = it.cpu().numpy()
    logp, lse, entropy, ai, al = rs.route_logprobs(logits, it, alternatives=k)
    counts, tokens_, sums, loss = rs.route_balance(logits, it, coef=0.1)
    kl = rs.route_distill(logits, ai, al + 0.5)
    assert not any(v.requires_grad for v in (logp, lse, entropy, al, sums, loss, kl))
    g, gz = rng.normal(size=(T, k)).astype(np.float32), rng.normal(size=T).astype(np.float32)
    grad = rs.route_logprobs_backward(logits, it, _dev(g), _dev(gz))
    rs.route_balance_backward(logits, k, counts, tokens_, torch.ones_like(loss), coef=0.1, accumulate=True, out=grad)
    rs.route_distill_backward(logits, ai, al + 0.5, torch.ones_like(kl), accumulate=True, out=grad)
    assert not grad.requires_grad
    logits.backward(grad)
    a, sa = R.logprobs_backward(x, idx, g.astype(float), gz.astype(float), np.zeros(T))
    c = R.balance(x, idx, [(0, T)], 0.1)
    b, sb = R.balance_backward(x, k, [(0, T)], 0.1, c[0], c[1], np.ones(1))
    d, sd = R.distill_backward(x, ai.cpu().numpy(), (al + 0.5).double().cpu().numpy(), np.ones(T))
    want = (a + b + d).T @ tokens.astype(float)
    # the gradient's error, 4 delta of its terms' magnitudes with t up to 2 Z, through the product, which adds T terms in fp32
    size = (sa + sb + sd)
    off = (size * (4 * _delta(x, 1.0)[:, None] + (5 * np.abs(x).max() + 8) * U)).T @ np.abs(tokens) + T * U * (np.abs(a + b + d).T @ np.abs(tokens))
    _near(w.grad, want, off, "gradient of the gate")


def _cuts(rng, T, groups, ragged):
    if not ragged:
        return np.arange(groups + 1) * (T // groups)
    return np.sort(rng.integers(0, T + 1, size=groups + 1))


SUMS = [  # rows, experts, groups, ragged: one record a group and many, one tile of columns and several, workgroups of 256 and 512 threads
    (400_000, 2, 2, True), (400_000, 7, 2, True), (400_000, 7, 1500, True), (262_144, 8, 4, False), (262_144, 8, 1, False), (4096 * 37, 8, 4096, False),
    (137_000, 61, 150, True), (137_500, 61, 1, False), (100_000, 100, 20, True), (60_000, 256, 3, True), (65_536, 256, 1, False), (27_900, 300, 150, True),
    (9_000, 891, 7, True), (8_192, 1024, 2, False), (1_000, 1024, 40, True)]


@pytest.mark.parametrize("T,E,groups,ragged", SUMS)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_no_row_is_lost_in_the_sums(T, E, groups, ragged, dtype):
    """Rows with one expert left have p = 1 there, and whole numbers below 2^24 add up exactly in any order: prob_sum is the number of rows."""
    rng = np.random.default_rng(T + E)
    cuts = _cuts(rng, T, groups, ragged)
    left = rng.integers(0, E, size=T)
    counted = rng.random(T) >= 0.1
    x = torch.full((T, E), -float("inf"), dtype=TYPES[dtype], device=DEV)
    x[torch.arange(T, device=DEV), _dev(left)] = _dev(rng.normal(size=T) * 3).to(TYPES[dtype])
    x[_dev(~counted)] = float("nan")
    picks = _dev(((left + 1) % E).astype(np.int32)).view(T, 1)
    args = dict(group_off=_dev(cuts)) if ragged else dict(groups=groups)
    counts, tokens, sums, loss = rs.route_balance(x, picks, row_mask=_dev(counted.astype(np.uint8)), **args)
    group = np.searchsorted(cuts, np.arange(T), side="right") - 1
    use = counted & (group >= 0) & (group < groups)
    want = np.bincount(group[use] * E + left[use], minlength=groups * E).reshape(groups, E)
    np.testing.assert_array_equal(sums.double().cpu().numpy(), want.astype(float))
    np.testing.assert_array_equal(tokens.cpu().numpy(), want.sum(axis=1))
    np.testing.assert_array_equal(counts.cpu().numpy(), np.roll(want, 1, axis=1))
    n = np.maximum(want.sum(axis=1), 1).astype(float)
    exact = E / (n * n) * (np.roll(want, 1, axis=1) * want).sum(axis=1)             # formed in fp64, rounded once
    _near(loss, exact, exact * 2 * U, "loss")


def test_sums_beyond_2_24():
    """Where fp32 no longer holds every whole number the parts are added up in more bits, and the sum is rounded once."""
    T = (1 << 25) + 1001
    x = torch.full((T, 2), -float("inf"), dtype=torch.bfloat16, device=DEV)
    left = torch.zeros(T, dtype=torch.int64, device=DEV)
    left[::3] = 1
    x.scatter_(1, left.view(T, 1), 0.5)
    counts, tokens, sums, loss = rs.route_balance(x, left.to(torch.int32).view(T, 1))
    want = torch.bincount(left, minlength=2)
    assert torch.equal(counts[0], want) and int(tokens) == T and torch.equal(sums[0], want.double().float())
    exact = 2.0 / float(T) ** 2 * float((want.double() ** 2).sum())
    assert abs(float(loss) - exact) <= 2 * U * exact


@pytest.mark.parametrize("T,E,groups,ragged", SUMS)
def test_sums_by_the_length_of_their_chains(T, E, groups, ragged):
    """fp32 additions are the rounds of a workgroup only: at least 512 workgroups of at least 4 rows share all rows (or one has a group of at most 16384 logits), then 6 steps over lanes and 7 over
    wavefronts; the parts are added in fp64."""
    rng = np.random.default_rng(T + E + 1)
    cuts = _cuts(rng, T, groups, ragged)
    xt, x = _logits(rng, T, E, torch.float32)
    it, idx = _picks(rng, T, E, 2)
    args = dict(group_off=_dev(cuts)) if ragged else dict(groups=groups)
    counts, tokens, sums, loss = rs.route_balance(xt, it, **args)
    wc, wn, ws, wl = R.balance(x, idx, list(zip(cuts[:-1], cuts[1:])), 1.0)
    chain = max(-(-T // 2048), 0 if ragged else -(-min(T // groups, 16384 // E) // 4)) + 16
    worst = _delta(x, 1.0).max() + (2.5 / np.e + chain) * U
    # p's own error has 2.5 |t| u of itself: p |t| is at most 1/e of the row's, whose share of ws is not known: as many rows as there are
    _near(sums, ws, worst * ws + 2.5 / np.e * wn[:, None] * U, "prob_sum")
