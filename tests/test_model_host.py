"""What the model operators refuse before they touch a device, and the helpers that need none."""
import ctypes
import math

import pytest
import torch

from paper_2202_13538_amd import binding

P = 0x10000  # an aligned address that nothing reads: every call here is refused


def attention_args(**changes):
    a = dict(d_q=P, d_k=P, d_v=P, q_row=64, q_head=32, k_row=32, k_head=32, v_row=32, v_head=32, d_q_off=P, d_k_off=P,
             n_seqs=3, n_q=10, n_k=12, type=binding.BF16, heads=2, kv_heads=1, dim=32, causal=0, scale=0.2, d_bias=None,
             d_bucket=None, n_buckets=0, reach=0)
    assert set(changes) <= set(a)
    return binding.AttentionArgs(**(a | changes))


ATTENTION = [
    (binding.E_RANGE, dict(type=2)), (binding.E_RANGE, dict(type=-1)), (binding.E_RANGE, dict(n_seqs=-1)),
    (binding.E_RANGE, dict(n_q=-1)), (binding.E_RANGE, dict(n_k=binding.MAX_ROWS + 1)),
    (binding.E_RANGE, dict(n_q=binding.MAX_ROWS + 1)), (binding.E_RANGE, dict(dim=0)), (binding.E_RANGE, dict(dim=12)),
    (binding.E_RANGE, dict(dim=136)), (binding.E_RANGE, dict(heads=0)), (binding.E_RANGE, dict(kv_heads=0)),
    (binding.E_RANGE, dict(heads=3, kv_heads=2)), (binding.E_RANGE, dict(heads=65536)),
    (binding.E_RANGE, dict(q_row=63)), (binding.E_RANGE, dict(k_head=-8)),
    (binding.E_RANGE, dict(v_row=binding.MAX_STRIDE + 8)), (binding.E_RANGE, dict(scale=0.0)),
    (binding.E_RANGE, dict(scale=-1.0)), (binding.E_RANGE, dict(scale=math.nan)), (binding.E_RANGE, dict(scale=math.inf)),
    (binding.E_RANGE, dict(causal=2)), (binding.E_NULL, dict(d_bias=P)), (binding.E_NULL, dict(d_bucket=P)),
    (binding.E_RANGE, dict(d_bias=P, d_bucket=P, n_buckets=0)),
    (binding.E_RANGE, dict(d_bias=P, d_bucket=P, n_buckets=4, reach=binding.MAX_REACH + 1)),
    (binding.E_RANGE, dict(d_bias=P, d_bucket=P, n_buckets=4, reach=-1)), (binding.E_NULL, dict(d_q_off=None)),
    (binding.E_NULL, dict(d_k_off=None)), (binding.E_NULL, dict(d_q=None)), (binding.E_NULL, dict(d_k=None)),
    (binding.E_NULL, dict(d_v=None)), (binding.E_RANGE, dict(d_q=P + 8)), (binding.E_RANGE, dict(d_v=P + 2)),
    (binding.E_RANGE, dict(n_seqs=0)), (binding.E_CTX, {}),
]


@pytest.mark.parametrize("status,changes", ATTENTION, ids=lambda x: str(x))
def test_attention_refuses(status, changes):
    lib = binding.load()
    assert lib.surel_attention(None, ctypes.byref(attention_args(**changes)), P, P) == status


def test_attention_refuses_no_arguments():
    assert binding.load().surel_attention(None, None, P, P) == binding.E_NULL


def test_binding_refuses_tensors_that_do_not_fit():
    t = torch.zeros(4, 2, 32)
    with pytest.raises(TypeError, match="bfloat16 or torch.float16"):
        binding.attention(None, t, t, t, torch.tensor([0, 4]))
    with pytest.raises(ValueError, match="GPU"):
        binding.attention(None, t.half(), t.half(), t.half(), torch.tensor([0, 4]))


@pytest.mark.parametrize("reach,buckets,causal", [(0, 1, True), (0, 2, False), (1, 2, True), (15, 16, True),
                                                  (128, 32, False), (128, 32, True), (1024, 64, False), (5, 40, True)])
def test_distance_buckets(reach, buckets, causal):
    got = binding.distance_buckets(reach, buckets, causal)
    assert len(got) == 2 * reach + 1 and min(got) == 0 and max(got) < buckets
    half = buckets if causal else buckets // 2
    back, ahead = got[:reach + 1][::-1], got[reach:]       # by |distance|
    assert back == sorted(back) and max(back) < half
    near = max(1, half // 2)
    for d in range(reach + 1):
        want = d if d < near else min(half - 1, near + math.floor(
            (half - near) * math.log(d / near) / math.log(reach / near) + 1e-9)) if reach > near else min(near, half - 1)
        assert back[d] == want, d
        if d:
            assert ahead[d] == (want if causal else half + want)


def test_distance_buckets_refuse():
    for bad in ((-1, 4, True), (4, 0, True), (4, 1, False)):
        with pytest.raises(ValueError):
            binding.distance_buckets(*bad)
