"""Offsets beyond 32 bits: a 4-bit weight just below the 2 GiB that a buffer may have, activations and outputs
whose elements pass 2^31, and a block residual over more than 2^31 elements, against 64 bits where they end."""
import pytest
import torch

import __graft_entry__ as graft
from test_block_residual import close, kwargs, terms
from test_w4 import EPS, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 64 GB of free GPU memory")
    return flashnorm


def test_a_weight_of_almost_two_gigabytes(fn):
    K, N, G = 65536, 60000, 128
    assert 2.08e9 < fn.lib().fold_weights_w4_size(K, N, 0, G) < 2 ** 31
    gen = torch.Generator(DEV).manual_seed(1)
    codes = torch.randint(0, 16, (K, N), generator=gen, dtype=torch.uint8, device=DEV)
    scales = ((torch.rand(K // G, N, generator=gen, device=DEV) + 0.5) * K ** -0.5 / 4).to(torch.bfloat16)
    zeros = torch.randint(0, 16, (K // G, N), generator=gen, dtype=torch.uint8, device=DEV)
    w4 = fn.pack_weights_w4(codes, scales, zeros, group=G)
    for M in (2, 16, 40, 130):
        a = torch.randn(M, K, generator=gen, device=DEV).to(torch.bfloat16)
        y = fn.flashnorm_linear_w4(a, w4, EPS)
        for n in (0, N // 2, N - 50):
            cols = slice(n, n + 50)
            s = scales[:, cols].double().repeat_interleave(G, 0)
            W = (codes[:, cols].double() - zeros[:, cols].double().repeat_interleave(G, 0)) * s
            x = a.double()
            r = (EPS + x.square().mean(1, keepdim=True)).rsqrt()
            ref = (x @ W) * r
            mag = (2.0 ** -13 * (x.abs() @ (8.0 * s.abs())) + 1.5 * 2.0 ** -11 * (x.abs() @ W.abs())) * r
            check(y[:, cols], ref.cpu(), (2.0 ** -8 * ref.abs() + mag).cpu(), (M, n))


def test_rows_whose_elements_pass_two_to_the_31(fn):
    """Activations and outputs with pitches that put the last rows beyond 2^31 elements."""
    M, K, N, ld = 1100, 256, 48, 1 << 21
    gen = torch.Generator(DEV).manual_seed(2)
    codes = torch.randint(0, 16, (K, N), generator=gen, dtype=torch.uint8, device=DEV)
    scales = ((torch.rand(K // 64, N, generator=gen, device=DEV) + 0.5) / 64).to(torch.bfloat16)
    w4 = fn.pack_weights_w4(codes, scales, group=64)
    W = (codes.double() - 8.0) * scales.double().repeat_interleave(64, 0)
    a = torch.empty(M, ld, dtype=torch.bfloat16, device=DEV)[:, :K]
    out = torch.empty(M, ld, dtype=torch.bfloat16, device=DEV)[:, :N]
    a.copy_(torch.randn(M, K, generator=gen, device=DEV))
    fn.flashnorm_linear_w4(a, w4, EPS, out=out)
    x = a.double()
    r = (EPS + x.square().mean(1, keepdim=True)).rsqrt()
    ref = (x @ W) * r
    T = 8.0 * scales.double().abs().repeat_interleave(64, 0)
    mag = (2.0 ** -13 * (x.abs() @ T) + 1.5 * 2.0 ** -11 * (x.abs() @ W.abs())) * r
    check(out, ref.cpu(), (2.0 ** -8 * ref.abs() + mag).cpu(), "all rows")
    fn.flashnorm_linear_w4(a[-5:], w4, EPS, out=out[-5:])  # the few-row kernel, at the end of the buffer
    check(out[-5:], ref[-5:].cpu(), (2.0 ** -8 * ref.abs() + mag)[-5:].cpu(), "last rows")


def test_a_block_residual_of_more_than_two_to_the_31_elements(fn):
    M, K = 132000, 16384
    assert M * K > 2 ** 31
    gen = torch.Generator(DEV).manual_seed(3)
    big = lambda: torch.empty(M, K, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    v = {"x": big(), "h": big(), "g_post": torch.rand(K, generator=gen, device=DEV) + 0.5,
         "g_pre": torch.rand(K, generator=gen, device=DEV) + 0.5}
    kw = kwargs(v, 0, 1.0, 0.5)
    out, normed = fn.flashnorm_block_residual(v["x"], v["h"], **kw)
    rows = [0, 1, M // 2, M - 2, M - 1]
    part = {n: (t[rows] if t.dim() == 2 else t).cpu() for n, t in v.items()}
    d, p, gp, z, gate, ref, mag, r = terms(part, 0, 1.0, 0.5)
    close(out[rows], ref, 2.0 ** -8 * ref.abs() + 2.0 ** -17 * mag, "out")
    n = ref * r * d["g_pre"]
    # r's relative error: 2^-17 (1 + sum |mag ref| / sum ref^2), and that quotient is below 2 for such rows
    close(normed[rows], n, 2.0 ** -8 * n.abs() + 2.0 ** -15 * (mag * r) * d["g_pre"], "normed")
    del out
    # The gradients of the last rows do not depend on the others: as in a call of their own.
    dx, dh, _, dg_post, dg_pre = fn.flashnorm_block_residual_bwd(v["x"], v["h"], v["h"], normed, **kw)
    one = [t[-3:].contiguous() for t in (v["x"], v["h"], v["h"], normed)]
    dx1, dh1, *_ = fn.flashnorm_block_residual_bwd(*one, **kw)
    assert torch.equal(dx[-3:], dx1) and torch.equal(dh[-3:], dh1)
    assert torch.isfinite(dg_post).all() and torch.isfinite(dg_pre).all()
