"""The operators on a router's logits where their arguments are at the edge of what the header allows.  Tolerances as derived in test_gpu_router.py."""
import numpy as np
import pytest
import torch

from oracle import router as R
from test_gpu_router import DEV, TYPES, U, _delta, _dev, _gradient_near, _logits, _near

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
