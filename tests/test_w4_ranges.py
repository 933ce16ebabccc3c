"""4-bit products whose columns hold scales that lie far apart, and where the small ones alone count.

Tolerance of the many-row kernel before the output's rounding (n: the power of two that brings the column's largest
scale S into [2^9, 2^10)): a group's scale s n and a weight (q - z) s n are rounded to fp16, each by 2^-12 of
itself or, below fp16's normal numbers, by 2^-25, so a weight is off by 2^-11 of itself + (|q - z| + 1) 2^-25 / n, and with
|q - z| <= 15 the latter is at most 2^-21 / n <= 2^-30 S.  fp32 sums of terms of both signs: 16 roundings of 2^-24 of A."""
import pytest
import torch

import __graft_entry__ as graft
from test_w4_shapes import plan

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return flashnorm


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("exponent", [-12, -18, -20, -22, -24, -27, -32])
def test_small_scales_beside_large_ones(fn, exponent, alike, group):
    """The groups of large scales meet zeros in a: the output is what the small ones give, codes of even and of odd places
    against each other, so that an error of one kind shows (most where a column's groups are alike but for a power of
    two, and round alike)."""
    M, K, N = 300, 1024, 5000
    assert plan(M, K, N, False, group, False).many
    gen = torch.Generator(DEV).manual_seed(group - exponent)
    big = (torch.arange(K, device=DEV) // group) % 4 == 0
    S = torch.exp2(torch.randint(-3, 4, (1, N), generator=gen, device=DEV).float())
    scales = (1.0 + torch.rand(K // group, N, generator=gen, device=DEV)).to(torch.bfloat16).float()
    if alike:
        scales = scales[:1].expand(K // group, N)
    scales = scales * S * torch.where(big[::group, None], 1.0, 2.0 ** exponent)
    up = torch.randint(9, 16, (K, N), generator=gen, device=DEV, dtype=torch.uint8)
    odd = ((torch.arange(K, device=DEV) % 8) // 2 % 2 == 1)[:, None]
    codes = torch.where(odd, 16 - up, up)  # q - 8: 1..7 at k % 8 in 0, 1, 4, 5, and -7..-1 at 2, 3, 6, 7
    a = torch.rand(M, K, generator=gen, device=DEV) + 0.5
    a[:, big] = 0.0
    a = a.to(torch.bfloat16)
    w4 = fn.pack_weights_w4(codes, scales, group=group)
    y = fn.rowscale_linear_w4(a, w4).double()
    s = scales.double().repeat_interleave(group, 0)
    W = (codes.double() - 8.0) * s
    ref, A = a.double() @ W, a.double().abs() @ W.abs()
    top = s.amax(0)
    tol = 2.0 ** -8 * ref.abs() + 2.0 ** -11 * A + 16 * 2.0 ** -24 * A + 2.0 ** -30 * a.double().sum(1, keepdim=True) * top
    over = (y - ref).abs() / tol
    assert torch.isfinite(y).all() and over.max() <= 1, float(over.max())


@pytest.mark.parametrize("M", [3, 20, 300])
def test_rows_far_from_one(fn, M):
    """Rows of 2^-116 to 2^100, their subnormal bf16 values among them, through a weight of about one: 2^-13 of
    8 sum |a s| and 1.5 * 2^-11 of sum |a w| as in test_w4.py, and half a step of the output's subnormals."""
    K, N, group = 1024, 5000 if M == 300 else 200, 64
    assert plan(M, K, N, False, group, False).many == (M == 300)
    gen = torch.Generator(DEV).manual_seed(M)
    codes = torch.randint(0, 16, (K, N), generator=gen, device=DEV, dtype=torch.uint8)
    scales = (torch.rand(K // group, N, generator=gen, device=DEV) + 0.5).to(torch.bfloat16)
    e = torch.tensor([-116, -100, -60, 0, 60, 100], device=DEV)[torch.arange(M, device=DEV) % 6]
    a = (torch.randn(M, K, generator=gen, device=DEV).double() * torch.exp2(e.double())[:, None]).to(torch.bfloat16)
    scale = torch.rand(M, generator=gen, device=DEV) + 0.5
    w4 = fn.pack_weights_w4(codes, scales, group=group)
    s = scales.double().repeat_interleave(group, 0)
    W = (codes.double() - 8.0) * s
    for rs in (None, scale):
        y = fn.rowscale_linear_w4(a, w4, row_scale=rs)
        f = torch.ones(M, 1, dtype=torch.float64, device=DEV) if rs is None else rs.double()[:, None]
        x = a.double()
        ref = (x @ W) * f
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -13 * (x.abs() @ (8.0 * s)) + 1.5 * 2.0 ** -11 * (x.abs() @ W.abs())) * f + 2.0 ** -134
        over = (y.double() - ref).abs() / tol
        assert torch.isfinite(y).all() and over.max() <= 1, float(over.max())


@pytest.mark.parametrize("M", [3, 20, 300])
@pytest.mark.parametrize("rows,scales_at,row_scale", [(100, -80, 50), (-60, 80, -60), (90, 0, -100), (-100, 60, 100), (0, -70, 120)])
def test_row_scales_far_from_one(fn, rows, scales_at, row_scale, M):
    """A row's values, the weight's scales and the row's scale far from one, and the output near it."""
    K, N, group = 1024, 5000 if M == 300 else 200, 32
    gen = torch.Generator(DEV).manual_seed(M)
    codes = torch.randint(0, 16, (K, N), generator=gen, device=DEV, dtype=torch.uint8)
    scales = ((torch.rand(K // group, N, generator=gen, device=DEV) + 0.5) * 2.0 ** scales_at).to(torch.bfloat16)
    a = (torch.randn(M, K, generator=gen, device=DEV).clamp(-1, 1) * 2.0 ** rows).to(torch.bfloat16)
    scale = (torch.rand(M, generator=gen, device=DEV) + 0.5) * 2.0 ** row_scale
    w4 = fn.pack_weights_w4(codes, scales, group=group)
    y = fn.rowscale_linear_w4(a, w4, row_scale=scale)
    s = scales.double().repeat_interleave(group, 0)
    W, x, f = (codes.double() - 8.0) * s, a.double(), scale.double()[:, None]
    ref = (x @ W) * f
    tol = 2.0 ** -8 * ref.abs() + (2.0 ** -13 * (x.abs() @ (8.0 * s)) + 1.5 * 2.0 ** -11 * (x.abs() @ W.abs())) * f
    over = (y.double() - ref).abs() / tol
    assert torch.isfinite(y).all() and over.max() <= 1, float(over.max())
