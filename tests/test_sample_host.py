"""What surel_sample_classes refuses before it touches a device."""
import types

import pytest
import torch

from paper_2202_13538_amd import binding

P = 0x10000  # an aligned address that nothing reads: every call here is refused
R, N, C = binding.E_RANGE, binding.E_NULL, binding.E_CTX
CALL = dict(type=binding.BF16, logits=P, row=100, rows=5, classes=100, u=P, temperature=P, top_k=P, top_p=P, min_p=P, chosen=P,
            logp=P)


@pytest.mark.parametrize("status,changes", [
    (R, dict(type=-1)), (R, dict(type=3)), (R, dict(rows=-1)), (R, dict(rows=binding.MAX_ROWS + 1)), (R, dict(classes=0)),
    (R, dict(classes=binding.MAX_NODES + 1)), (R, dict(row=-1)), (R, dict(row=2 ** 40 + 1)), (N, dict(logits=None)),
    (N, dict(u=None)), (N, dict(chosen=None)), (N, dict(logp=None)), (R, dict(logits=P + 1)),
    (R, dict(type=binding.FP32, logits=P + 2)), (C, {}), (C, dict(temperature=None, top_k=None, top_p=None, min_p=None)),
    (C, dict(logits=P + 2)), (C, dict(type=binding.FP32, logits=P + 4)), (C, dict(rows=1, row=2 ** 50)),
    (C, dict(rows=0, logits=None, u=None, chosen=None, logp=None))], ids=str)
def test_sample_refuses(status, changes):
    assert binding.load().surel_sample_classes(None, *(CALL | changes).values()) == status


def test_binding_refuses_tensors_that_do_not_fit():
    ctx = types.SimpleNamespace(handle=None, device=torch.device("cuda", 0), stream=None)
    z, u = torch.zeros(3, 5), torch.zeros(3)
    with pytest.raises(TypeError, match="float32"):
        binding.sample_classes(ctx, z.double(), u)
    with pytest.raises(ValueError, match="GPU"):
        binding.sample_classes(ctx, z, u)
