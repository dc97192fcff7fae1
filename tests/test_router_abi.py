"""Argument checks of the operators on a router's logits: on the host, before anything is launched."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2510_19262_amd as rs

P = C.c_void_p
A, B, D = P(0x1000), P(0x2000), P(0x3000)     # never dereferenced: validation fails first
NAN, INF = float("nan"), float("inf")


def test_dtype_codes_are_the_headers():
    from paper_2510_19262_amd import binding
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "railsched.h")).read()
    assert re.search(r"RAILSCHED_F32 = 0, RAILSCHED_BF16 = 1, RAILSCHED_F16 = 2", header)
    assert binding.DTYPES == {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


# (dtype, rows, E, ld) that no operator takes, and why
HEADS = [((-1, 4, 8, 8), -1), ((3, 4, 8, 8), -1), ((0, -1, 8, 8), -1), ((0, 4, 0, 8), -1), ((0, 4, 8, 7), -1), ((0, 4, 1025, 1025), -3),
         ((0, 1 << 31, 8, 8), -3), ((0, 4, 8, (1 << 31) + 1), -3)]


@pytest.mark.parametrize("head,want", HEADS)
def test_heads(head, want):
    lib = rs.load()
    dt, rows, E, ld = head
    big = 1 << 40
    assert lib.railsched_route_logprobs(A, dt, rows, E, ld, 1.0, None, B, 2, 0, D, None, None, None, None, None) == want
    assert lib.railsched_route_logprobs_backward(A, dt, rows, E, ld, 1.0, None, B, 2, D, None, None, 0, B, big, None) == want
    assert lib.railsched_route_balance(A, dt, rows, E, ld, None, B, 2, None, 1, 1.0, D, D, D, D, A, big, None) == want
    assert lib.railsched_route_balance_backward(A, dt, rows, E, ld, None, 2, None, 1, 1.0, D, D, D, 0, B, big, None) == want
    assert lib.railsched_route_distill(A, dt, rows, E, ld, 1.0, None, B, D, None, 2, D, None) == want
    assert lib.railsched_route_distill_backward(A, dt, rows, E, ld, 1.0, None, B, D, None, 2, D, 0, B, big, None) == want


@pytest.mark.parametrize("tau", [0.0, -1.0, NAN, INF, 2.0 ** 61, 2.0 ** -61])
def test_temperature(tau):
    lib = rs.load()
    assert lib.railsched_route_logprobs(A, 0, 4, 8, 8, tau, None, B, 2, 0, D, None, None, None, None, None) == -1
    assert lib.railsched_route_logprobs_backward(A, 0, 4, 8, 8, tau, None, B, 2, D, None, None, 0, B, 8, None) == -1
    assert lib.railsched_route_distill(A, 0, 4, 8, 8, tau, None, B, D, None, 2, D, None) == -1
    assert lib.railsched_route_distill_backward(A, 0, 4, 8, 8, tau, None, B, D, None, 2, D, 0, B, 8, None) == -1


def test_logprobs_validation():
    f = rs.load().railsched_route_logprobs   # (logits, dtype, rows, E, ld, tau, mask, idx, k, m, logp, lse, entropy, alt_idx, alt_logp, stream)
    assert f(None, 0, 4, 8, 8, 1.0, None, B, 2, 0, D, None, None, None, None, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 9, 0, D, None, None, None, None, None) == -1
    assert f(A, 0, 4, 8, 8, 1.0, None, B, -1, 0, D, None, None, None, None, None) == -1
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, 9, D, None, None, D, D, None) == -1
    assert f(A, 0, 4, 128, 128, 1.0, None, B, 2, 65, D, None, None, D, D, None) == -3
    assert f(A, 0, 4, 8, 8, 1.0, None, None, 2, 0, D, None, None, None, None, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, 0, None, None, None, None, None, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, 3, D, None, None, None, D, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, 3, D, None, None, D, None, None) == -2
    assert f(None, 0, 0, 8, 8, 1.0, None, None, 2, 3, None, None, None, None, None, None) == 0       # nothing to do


def test_gradient_validation():
    f = rs.load().railsched_route_logprobs_backward   # (logits, dtype, rows, E, ld, tau, mask, idx, k, d_logp, d_lse, d_entropy, add, d_logits, ld_d, stream)
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, D, None, None, 0, None, 8, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, D, None, None, 0, A, 8, None) == -1                     # in place
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, D, None, None, 2, B, 8, None) == -1
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, D, None, None, 0, B, 7, None) == -1
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 2, D, None, None, 0, B, (1 << 31) + 1, None) == -3
    assert f(A, 0, 4, 8, 8, 1.0, None, None, 2, D, None, None, 0, B, 8, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, 9, D, None, None, 0, B, 8, None) == -1
    assert f(None, 0, 0, 8, 8, 1.0, None, None, 2, None, None, None, 0, None, 8, None) == 0


def test_balance_validation():
    lib = rs.load()
    need = lib.railsched_route_balance_workspace_bytes(1000, 4, 8)
    assert need > 0 and need % 256 == 0
    assert lib.railsched_route_balance_workspace_bytes(0, 0, 8) % 256 == 0
    for bad in ((-1, 4, 8), (1000, -1, 8), (1000, 4, 0), (1000, 4, 1025), (1 << 31, 4, 8)):
        assert lib.railsched_route_balance_workspace_bytes(*bad) == 0
    f = lib.railsched_route_balance   # (logits, dtype, rows, E, ld, mask, idx, k, off, groups, coef, counts, tokens, prob_sum, loss, ws, ws_bytes, stream)
    ok = [A, 0, 1000, 8, 8, None, B, 2, None, 4, 1.0, D, D, D, D, A, need, None]

    def call(**kw):
        names = "logits dtype rows E ld mask idx k off groups coef counts tokens prob_sum loss ws ws_bytes stream".split()
        return f(*[kw.get(n, v) for n, v in zip(names, ok)])

    assert call(logits=None) == -2 and call(idx=None) == -2
    assert call(k=0) == -1 and call(k=9) == -1 and call(groups=-1) == -1
    assert call(groups=3) == -1                                              # 1000 rows in three equal parts
    assert call(groups=0) == -1                                              # rows, but no group
    assert call(off=D, groups=(1 << 23) + 1) == -3 and lib.railsched_route_balance_workspace_bytes(1000, (1 << 23) + 1, 8) == 0
    for n in ("counts", "tokens", "prob_sum", "loss"):
        assert call(**{n: None}) == -2
    assert call(ws=None) == -5 and call(ws_bytes=need - 1) == -5 and call(ws=P(0x1010)) == -5
    assert call(rows=0, groups=0) == 0 and call(off=D, groups=0) == 0
    b = lib.railsched_route_balance_backward   # (logits, dtype, rows, E, ld, mask, k, off, groups, coef, counts, tokens, d_loss, add, d_logits, ld_d, stream)
    assert b(A, 0, 1000, 8, 8, None, 0, None, 4, 1.0, D, D, D, 0, B, 8, None) == -1
    assert b(A, 0, 1000, 8, 8, None, 2, None, 3, 1.0, D, D, D, 0, B, 8, None) == -1
    assert b(A, 0, 1000, 8, 8, None, 2, None, 4, 1.0, None, D, D, 0, B, 8, None) == -2
    assert b(A, 0, 1000, 8, 8, None, 2, None, 4, 1.0, D, None, D, 0, B, 8, None) == -2
    assert b(A, 0, 1000, 8, 8, None, 2, None, 4, 1.0, D, D, None, 0, B, 8, None) == -2
    assert b(A, 0, 1000, 8, 8, None, 2, None, 4, 1.0, D, D, D, 0, A, 8, None) == -1
    assert b(A, 0, 1000, 8, 8, None, 2, None, 4, 1.0, D, D, D, 3, B, 8, None) == -1
    assert b(A, 0, 1000, 8, 8, None, 2, None, 4, 1.0, D, D, D, 0, B, 7, None) == -1
    assert b(None, 0, 0, 8, 8, None, 2, None, 4, 1.0, None, None, None, 0, None, 8, None) == 0


def test_distill_validation():
    lib = rs.load()
    f = lib.railsched_route_distill   # (logits, dtype, rows, E, ld, tau, mask, t_idx, t_logit, t_lse, K, loss, stream)
    assert f(None, 0, 4, 8, 8, 1.0, None, B, D, None, 2, D, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, None, D, None, 2, D, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, None, None, 2, D, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, D, None, 2, None, None) == -2
    assert f(A, 0, 4, 8, 8, 1.0, None, B, D, None, 0, D, None) == -1
    assert f(A, 0, 4, 8, 8, 1.0, None, B, D, None, 9, D, None) == -1
    assert f(A, 0, 4, 128, 128, 1.0, None, B, D, None, 65, D, None) == -3
    assert f(None, 0, 0, 8, 8, 1.0, None, None, None, None, 2, None, None) == 0
    b = lib.railsched_route_distill_backward   # (logits, dtype, rows, E, ld, tau, mask, t_idx, t_logit, t_lse, K, d_loss, add, d_logits, ld_d, stream)
    assert b(A, 0, 4, 8, 8, 1.0, None, B, D, None, 2, None, 0, B, 8, None) == -2
    assert b(A, 0, 4, 8, 8, 1.0, None, B, D, None, 2, D, 0, A, 8, None) == -1
    assert b(A, 0, 4, 8, 8, 1.0, None, B, D, None, 2, D, -1, B, 8, None) == -1
    assert b(A, 0, 4, 128, 128, 1.0, None, B, D, None, 65, D, 0, B, 128, None) == -3


def test_binding_rejects_host_tensors():
    x, i = torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32)
    for call in (lambda: rs.route_logprobs(x, i), lambda: rs.route_logprobs_backward(x, i), lambda: rs.route_balance(x, i),
                 lambda: rs.route_balance_backward(x, 2, i, i, i), lambda: rs.route_distill(x, i, x),
                 lambda: rs.route_distill_backward(x, i, x, x)):
        with pytest.raises(ValueError):
            call()
