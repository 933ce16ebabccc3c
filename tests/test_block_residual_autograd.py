"""The block residual beside torch's own autograd: outputs carry no gradient, and what a call writes counts as written."""
import pytest
import torch

import __graft_entry__ as graft

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return flashnorm


def test_a_tensor_that_is_written_counts_as_changed(fn):
    """torch refuses a backward pass through values that an in-place call has replaced since."""
    leaf = torch.randn(3, 64, device=DEV, requires_grad=True)
    h = leaf * 1.0
    x, g = torch.randn(3, 64, device=DEV), torch.ones(64, device=DEV)
    loss = (h * h).sum()  # keeps h
    with torch.no_grad():
        fn.flashnorm_block_residual(x, h, out=h)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    out, normed, inv = torch.empty_like(x), torch.empty_like(x), torch.empty(3, device=DEV)
    before = [t._version for t in (out, normed, inv, x)]
    fn.flashnorm_block_residual(x, h.detach(), g_pre=g, out=out, normed=normed, inv_rms=inv)
    assert [t._version for t in (out, normed, inv, x)] == [before[0] + 1, before[1] + 1, before[2] + 1, before[3]]


def test_products_count_what_they_write(fn):
    w4 = fn.fold_weights_w4(torch.randn(64, 32, device=DEV), group=32)
    big = fn.fold_weights_w4(torch.randn(1024, 8192, device=DEV), group=32)
    a = torch.randn(4, 64, device=DEV).to(torch.bfloat16)
    out, inv = torch.empty(4, 32, dtype=torch.bfloat16, device=DEV), torch.empty(4, device=DEV)
    before = out._version, inv._version, a._version
    fn.flashnorm_linear_w4(a, w4, 1e-6, out=out, inv_rms=inv)
    assert (out._version, inv._version, a._version) == (before[0] + 1, before[1] + 1, before[2])
    ws = torch.empty(fn.lib().flashnorm_w4_workspace_size(1000, 1024, 8192, 0, 32), dtype=torch.uint8, device=DEV)
    version = ws._version
    fn.rowscale_linear_w4(torch.randn(1000, 1024, device=DEV).to(torch.bfloat16), big, workspace=ws)
    assert ws._version == version + 1


def test_tensors_of_inference_mode(fn):
    with torch.inference_mode():
        x, h = torch.randn(3, 64, device=DEV), torch.randn(3, 64, device=DEV)
        want, _ = fn.flashnorm_block_residual(x, h)
        got, _ = fn.flashnorm_block_residual(x, h, out=h)
    assert got is h and torch.equal(want, h)
    fn.flashnorm_block_residual(x, h, out=h)  # an inference tensor, outside: it has no version


def test_outputs_carry_no_gradient(fn):
    """As documented: the gradients are a call of their own."""
    x, h = (torch.randn(3, 64, device=DEV, requires_grad=True) for _ in range(2))
    out, _ = fn.flashnorm_block_residual(x, h)
    assert not out.requires_grad
    assert "flashnorm_block_residual_bwd" in fn.flashnorm_block_residual.__doc__
    assert "autograd" in fn.flashnorm_block_residual.__doc__
