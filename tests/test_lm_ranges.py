"""CPU-only: parameters whose products leave float32's range are refused, where they would make a row's own maximum 0 * infinity."""
import math

import pytest

from paper_2012_15198_amd import cxlm as lm

SUFFIXES = ["", "_bf16", "_f16"]
A, B, C, D, E, F, G = (k << 28 for k in range(1, 8))                 # far apart, aligned; never handed to a kernel
LARGEST = 3.4028234663852886e38
LOG2E = math.log2(math.e)


@pytest.mark.parametrize("suffix", SUFFIXES)
@pytest.mark.parametrize("scale", [LARGEST / LOG2E * 1.0001, 2.9e38, LARGEST, math.inf])
def test_a_scale_whose_base_two_factor_overflows(suffix, scale):
    assert getattr(lm.lib(), "cx_token_scores" + suffix)(A, 50, 600, 50, B, scale, C, D, 4, E, F, None, 0, None) == -2


@pytest.mark.parametrize("suffix", SUFFIXES)
@pytest.mark.parametrize("tau,w_kl", [(4.2e-39, 1.0), (1e-45, 1.0), (2e38, 2.0), (1e20, 1e20)])
def test_a_temperature_whose_factors_overflow(suffix, tau, w_kl):
    head = (A, 50, 600, 50, 4, B, C, D, tau, w_kl, 0.5)
    assert getattr(lm.lib(), "cx_distill_loss" + suffix)(*head, E, F, None, 0, None) == -2
    assert getattr(lm.lib(), "cx_distill_grad" + suffix)(*head, F, E, G, 50, None) == -2
    assert getattr(lm.lib(), "cx_distill_step" + suffix)(*head, E, F, G, 50, None, 0, None) == -2
