"""Scales of gradients whose reciprocal times a logarithm of a sum leaves 32-bit floats are refused."""
import ctypes

import pytest

from paper_2202_13538_amd import binding
from test_model_host import P, attention_args


@pytest.mark.parametrize("scale,status", [(1e-30, binding.E_CTX), (7e-31, binding.E_RANGE), (1e-38, binding.E_RANGE), (1e-40, binding.E_RANGE)])
def test_smallest_scale_of_gradients(scale, status):
    args = attention_args(scale=scale)
    assert binding.load().surel_attention_grad(None, ctypes.byref(args), P, P, P, P, P, P, None) == status
    assert binding.load().surel_attention(None, ctypes.byref(args), P, P) == binding.E_CTX
