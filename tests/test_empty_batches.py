"""Batches without a token (no image among a step's inputs): rows as torch hands them over, forward and backward."""
import pytest
import torch

import paper_2505_17694_amd as C
from paper_2505_17694_amd.cache import _rows
from workloads import HeadConfig, DTYPE_BF16

DEV = "cuda:0"


def test_strides_of_no_tokens_say_nothing():
    """A sum's gradient is one number expanded: without a token it counts as contiguous, with strides of zero.  (On the CPU, whose
    index is -1.)"""
    got = []
    x = torch.zeros(0, 4, 64, dtype=torch.bfloat16, requires_grad=True)
    y = x * 1
    y.register_hook(got.append)
    y.sum().backward()
    g, = got
    assert g.stride() == (0, 0, 0) and g.is_contiguous()
    for t in (g, g.detach(), torch.zeros(64, 4, 0, dtype=torch.bfloat16).permute(2, 1, 0), torch.zeros(0, 4, 64, dtype=torch.bfloat16)):
        r = _rows(t, "g", t.shape, torch.bfloat16, -1)
        assert (r.data or 0, r.token_stride, r.head_stride) == (0, 0, 0)
    for bad in (g.float(), g[:, :3], torch.zeros(1, 64, 4, dtype=torch.bfloat16).transpose(1, 2)):      # one token's strides count
        with pytest.raises(ValueError):
            _rows(bad, "g", (len(bad), 4, 64), torch.bfloat16, -1)


@pytest.mark.gpu
@pytest.mark.parametrize("kw,positions", [(dict(), (0,)), (dict(axes=(16, 8, 8)), (3, 0)), (dict(axes=(16, 8, 8)), (0,)), (dict(blocks=2), (0,))])
@pytest.mark.parametrize("loss", ["sum", "mean", "grad", "twice"])
def test_gradients_of_no_tokens(kw, positions, loss):
    print(f"[case] no tokens {kw} {positions} {loss}", flush=True)
    rot = C.Rotary(64, device=DEV, **kw)
    at = torch.zeros(positions, dtype=torch.int64, device=DEV)
    x = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=DEV, requires_grad=True)
    y = rot.apply(x, at)
    assert y.shape == (0, 4, 64)
    if loss == "twice":
        w = torch.zeros_like(y, requires_grad=True)
        g, = torch.autograd.grad((y * w).sum(), x, create_graph=True)
        g.sum().backward()
        assert w.grad.shape == x.shape
    elif loss == "grad":
        y.backward(torch.zeros(64, 4, 0, dtype=torch.bfloat16, device=DEV).permute(2, 1, 0))
    else:
        getattr(y, loss)().backward()
    assert loss == "twice" or (x.grad.shape == x.shape and x.grad.dtype == x.dtype)
    # a leaf that only a part of the batch comes from: its gradient is whole
    leaf = torch.randn(5, 4, 64, device=DEV).bfloat16().requires_grad_()
    rot.apply(leaf[:0], at).sum().backward()
    assert leaf.grad.shape == leaf.shape and not leaf.grad.any()


@pytest.mark.gpu
def test_appends_of_no_tokens():
    cache = C.KVCache(HeadConfig(4, 2, 64, DTYPE_BF16), 4, device=DEV)
    none = torch.zeros(1, dtype=torch.bfloat16, device=DEV)
    at = torch.zeros(0, dtype=torch.int64, device=DEV)
    for rot in (None, C.Rotary(64, device=DEV), C.Rotary(64, device=DEV, axes=(16, 16))):
        out = cache.append(0, none.expand(0, 4, 64), none.expand(0, 2, 64), none.expand(0, 2, 64), at, at, rot)
        assert out.shape == (0, 4, 64)
