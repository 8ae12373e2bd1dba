"""Strides of attention's tensors that lead nowhere, of one row or one head, may be any."""
import ctypes

import pytest

from paper_2202_13538_amd import binding
from test_model_host import P, attention_args

ONE = [dict(n_q=1, q_row=63), dict(n_k=1, k_row=3, v_row=1 << 40), dict(heads=1, q_head=7), dict(k_head=1, v_head=33),
       dict(n_q=0, q_row=5), dict(n_k=0, k_row=9, v_row=11)]
MORE = [dict(n_q=2, q_row=63), dict(n_k=2, v_row=1 << 40), dict(heads=2, q_head=7), dict(heads=4, kv_heads=2, k_head=12),
        dict(n_q=1, q_row=-8), dict(heads=1, q_head=-1)]


@pytest.mark.parametrize("changes", ONE, ids=str)
def test_a_stride_that_leads_nowhere(changes):
    args = attention_args(**changes)   # (all that is left to refuse is the context)
    assert binding.load().surel_attention(None, ctypes.byref(args), P, P) == binding.E_CTX
    assert binding.load().surel_attention_grad(None, ctypes.byref(args), P, P, P, P, P, P, None) == binding.E_CTX


@pytest.mark.parametrize("changes", MORE, ids=str)
def test_a_stride_that_leads_somewhere(changes):
    args = attention_args(**changes)
    assert binding.load().surel_attention(None, ctypes.byref(args), P, P) == binding.E_RANGE
