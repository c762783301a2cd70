"""Temperatures whose inverse is no 32-bit number are refused before any launch."""
import pytest

from paper_2505_18719_gb300 import vla as V
from tests.test_lm_abi_cpu import grad, lib, logprobs, refused  # noqa: F401


@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 4e-39, -1e-39, -0.7, float("inf"), float("nan")])
def test_temperatures_that_are_refused(temperature):
    refused(logprobs(temperature=temperature), V.VLA_ERR_ARG, "vla_token_logprobs")
    refused(grad(temperature=temperature), V.VLA_ERR_ARG, "vla_token_logprobs_grad")


@pytest.mark.parametrize("temperature", [0.0, 5e-39, 2.0 ** -126, 1.0, 3e38])
def test_temperatures_that_are_taken(temperature):
    assert logprobs(temperature=temperature, rows=0) == V.VLA_OK
    assert grad(temperature=temperature, rows=0) == V.VLA_OK
