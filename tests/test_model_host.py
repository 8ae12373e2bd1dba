"""What the model operators refuse before they touch a device, and the helpers that need none."""
import ctypes
import math
import types

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


@pytest.mark.parametrize("status,changes", ATTENTION, ids=lambda x: str(x))
def test_attention_grad_refuses(status, changes):
    args = attention_args(**changes)
    dbias = P if args.d_bias else None
    assert binding.load().surel_attention_grad(None, ctypes.byref(args), P, P, P, P, P, P, dbias) == status


def test_outputs_that_are_missing_or_off_their_boundary():
    lib, plain = binding.load(), attention_args()
    biased = attention_args(d_bias=P, d_bucket=P, n_buckets=3, reach=1)
    fake = ctypes.create_string_buffer(4096)  # a context that is looked at only after these checks passed
    call = lambda args, *p: lib.surel_attention(fake, ctypes.byref(args), *p)  # noqa: E731
    assert call(plain, None, P) == call(plain, P, None) == binding.E_NULL
    assert call(plain, P + 8, P) == binding.E_RANGE
    call = lambda args, *p: lib.surel_attention_grad(fake, ctypes.byref(args), *p)  # noqa: E731
    for missing in range(6):
        assert call(plain, *[None if i == missing else P for i in range(6)], None) == binding.E_NULL
    for off in (0, 1, 3, 4, 5):
        assert call(plain, *[P + 8 if i == off else P for i in range(6)], None) == binding.E_RANGE
    assert call(plain, *[P] * 7) == binding.E_NULL          # a gradient of a bias that is not there
    assert call(biased, *[P] * 6, None) == binding.E_NULL


def test_attention_refuses_no_arguments():
    assert binding.load().surel_attention(None, None, P, P) == binding.E_NULL


LOSS = [  # status, changes of (type, h, w, labels, rows, classes, dim)
    (binding.E_RANGE, dict(type=2)), (binding.E_RANGE, dict(rows=-1)), (binding.E_RANGE, dict(rows=binding.MAX_ROWS + 1)),
    (binding.E_RANGE, dict(classes=0)), (binding.E_RANGE, dict(classes=binding.MAX_NODES + 1)),
    (binding.E_RANGE, dict(dim=0)), (binding.E_RANGE, dict(dim=20)), (binding.E_RANGE, dict(dim=264)),
    (binding.E_NULL, dict(h=None)), (binding.E_NULL, dict(w=None)), (binding.E_NULL, dict(labels=None)),
    (binding.E_RANGE, dict(h=P + 8)), (binding.E_RANGE, dict(w=P + 4)), (binding.E_CTX, {}),
]


@pytest.mark.parametrize("status,changes", LOSS, ids=lambda x: str(x))
def test_loss_refuses(status, changes):
    lib = binding.load()
    a = dict(type=binding.FP16, h=P, w=P, labels=P, rows=5, classes=100, dim=64) | changes
    shape = (a["rows"], a["classes"], a["dim"])
    assert lib.surel_softmax_loss(None, a["type"], a["h"], a["w"], a["labels"], *shape, P, P) == status
    assert lib.surel_softmax_loss_grad(None, a["type"], P, a["h"], a["w"], a["labels"], P, *shape, P, P) == status


def test_loss_outputs_that_are_missing_or_off_their_boundary():
    lib = binding.load()
    fake = ctypes.create_string_buffer(4096)
    for loss, lse in ((None, P), (P, None)):
        assert lib.surel_softmax_loss(fake, 0, P, P, P, 5, 100, 64, loss, lse) == binding.E_NULL
    call = lambda dloss, lse, dh, dw: lib.surel_softmax_loss_grad(fake, 0, dloss, P, P, P, lse, 5, 100, 64, dh, dw)  # noqa: E731
    for missing in range(4):
        assert call(*[None if i == missing else P for i in range(4)]) == binding.E_NULL
    assert call(P, P, P + 8, P) == call(P, P, P, P + 2) == binding.E_RANGE


def test_binding_refuses_tensors_that_do_not_fit():
    t = torch.zeros(4, 2, 32)
    with pytest.raises(TypeError, match="bfloat16 or torch.float16"):
        binding.attention(None, t, t, t, torch.tensor([0, 4]))
    with pytest.raises(ValueError, match="GPU"):
        binding.attention(None, t.half(), t.half(), t.half(), torch.tensor([0, 4]))
    h, w, labels = torch.zeros(3, 16).half(), torch.zeros(9, 16).half(), torch.zeros(3, dtype=torch.int32)
    for bad in ((h.float(), w, labels), (h, w.bfloat16(), labels), (h, w, labels.long())):
        with pytest.raises((TypeError, ValueError)):
            binding.softmax_loss(types.SimpleNamespace(handle=None), *bad)
    for bad in ((h[0], w, labels), (h, w[:, :8], labels), (h, w, labels[:2])):
        with pytest.raises(ValueError):
            binding.softmax_loss(types.SimpleNamespace(handle=None), *bad)


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


def test_reference_gradients_against_differences():
    """The gradients that the GPU's are held to, against central differences in 64 bits."""
    from attention_cases import inputs, reference
    q_lens, k_lens = [3, 1, 2], [4, 0, 7]
    q, k, v, q_off, k_off, how = inputs(q_lens, k_lens, 4, 2, 8, torch.float64, seed=1, reach=3, buckets=4,
                                        causal=True, device="cpu")
    g = torch.Generator().manual_seed(2)
    dout = torch.randn(q.shape, generator=g, dtype=torch.float64)
    r = reference(q, k, v, q_off, k_off, True, 0.3, dout=dout, **how)
    loss = lambda: (reference(q, k, v, q_off, k_off, True, 0.3, **how)["out"] * dout.numpy()).sum()  # noqa: E731
    h = 1e-5
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv"), (how["bias"], "dbias")):
        flat = x.view(-1)
        for i in torch.randperm(flat.numel(), generator=g)[:40].tolist():
            old = flat[i].item()
            flat[i] = old + h
            above = loss()
            flat[i] = old - h
            below = loss()
            flat[i] = old
            # the error of a central difference is h^2 / 6 of a third derivative of order one, and 1e-16 / h
            assert abs((above - below) / (2 * h) - r[name].reshape(-1)[i]) < 1e-8, (name, i)
