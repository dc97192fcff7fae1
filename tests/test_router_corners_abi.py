"""Argument checks of the operators on a router's logits at the edges of their limits: on the host, before anything is launched."""
import ctypes as C
import math

import pytest

import paper_2510_19262_amd as rs

P = C.c_void_p
A, B, D = P(0x1000), P(0x2000), P(0x3000)     # never dereferenced: validation fails first, or there are no rows


@pytest.mark.parametrize("tau", [2.0 ** -60, 1e-6, math.nextafter(2.0 ** -8, 0) * (1 - 2.0 ** -24), 2.0 ** 8 * (1 + 2.0 ** -23), 1e4, 2.0 ** 60])
def test_temperatures_that_distillation_does_not_take(tau):
    lib = rs.load()
    for rows in (4, 0):
        assert lib.railsched_route_distill(A, 0, rows, 8, 8, tau, None, B, D, None, 2, D, None) == -1
        assert lib.railsched_route_distill_backward(A, 0, rows, 8, 8, tau, None, B, D, None, 2, D, 0, B, 8, None) == -1


@pytest.mark.parametrize("tau", [2.0 ** -8, 0.1, 1.0, 100.0, 2.0 ** 8])
def test_temperatures_that_it_takes(tau):
    lib = rs.load()
    assert lib.railsched_route_distill(None, 0, 0, 8, 8, tau, None, None, None, None, 2, None, None) == 0
    assert lib.railsched_route_distill_backward(None, 0, 0, 8, 8, tau, None, None, None, None, 2, None, 0, None, 8, None) == 0


@pytest.mark.parametrize("tau", [2.0 ** -60, 2.0 ** 60])
def test_temperatures_of_the_others(tau):
    lib = rs.load()
    assert lib.railsched_route_logprobs(None, 0, 0, 8, 8, tau, None, None, 2, 0, None, None, None, None, None, None) == 0
    assert lib.railsched_route_logprobs_backward(None, 0, 0, 8, 8, tau, None, None, 2, None, None, None, 0, None, 8, None) == 0
