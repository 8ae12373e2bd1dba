"""Attention calls of more workgroups than a launch has are refused before a device is touched."""
import ctypes

import pytest

from paper_2202_13538_amd import binding
from test_model_host import P, attention_args


@pytest.mark.parametrize("changes", [dict(n_seqs=1 << 30, n_q=1 << 28, n_k=1 << 30, heads=2, kv_heads=2),
                                     dict(n_seqs=40_000, n_q=1 << 30, n_k=1 << 30, heads=65535, kv_heads=65535)])
def test_more_workgroups_than_a_launch_has(changes):
    lib, fake = binding.load(), ctypes.create_string_buffer(4096)   # (a context that only its number of compute units is read of)
    args = attention_args(k_row=512, v_row=512, q_row=512, **changes)
    assert lib.surel_attention(fake, ctypes.byref(args), P, P) == binding.E_RANGE
    assert lib.surel_attention_grad(fake, ctypes.byref(args), P, P, P, P, P, P, None) == binding.E_RANGE
