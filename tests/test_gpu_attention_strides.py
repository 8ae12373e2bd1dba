"""One row or one head, whose strides are not multiples of 8."""
import pytest
import torch

from attention_cases import offsets
from paper_2202_13538_amd import binding
from test_gpu_attention import BF, check
from test_gpu_attention_grad import check as check_gradients

pytestmark = pytest.mark.gpu


def test_strides_that_lead_nowhere():
    ctx = binding.Context(0)
    g = torch.Generator().manual_seed(1)
    some = torch.randn(8 * 4096, generator=g).to(BF).cuda()
    one_row = some.as_strided((1, 2, 32), (63, 40, 1))
    one_head = some.as_strided((50, 1, 32), (96, 7, 1))
    one_key = some.as_strided((1, 1, 32), (1 << 30, 5, 1))
    for q, k, q_lens, k_lens in ((one_row, one_head, [1], [50]), (one_head, one_head, [20, 30], [50, 0]), (one_row, one_key, [1], [1])):
        args = q, k, k, offsets(q_lens), offsets(k_lens), False, {}
        check(ctx, *args)
        check_gradients(ctx, *args)
    assert ctx.check() == 0
    ctx.close()
