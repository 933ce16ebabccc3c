"""The gradients of the block residual's norm weights over units of hundreds of rows and more than 2^31 elements, some
columns of them against sums in 64 bits over all rows.

Tolerance.  A unit of such widths has at most ceil(M / 512) rows, whose terms it adds one by one, and a workgroup adds the
units (or the pieces of a gate's rows) in 32 sums of 16 and those in turn: ceil(M / 512) + 48 additions, each off by
2^-24 of the sum of magnitudes at most; the terms' own errors are at most 2^-17 of their magnitudes
(tests/test_block_residual.py)."""
import pytest
import torch

import __graft_entry__ as graft
from test_block_residual import EPS_POST, EPS_PRE

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


@pytest.mark.parametrize("dtype,M,K,T", [(torch.bfloat16, 132000, 16384, 0), (torch.float32, 132000, 16384, 0),
                                         (torch.bfloat16, 600001, 4096, 777), (torch.float32, 1050000, 2056, 1 << 20)])
def test_norm_weights_and_gates(fn, dtype, M, K, T):
    assert M * K > 2 ** 31
    gen = torch.Generator(DEV).manual_seed(M)
    big = lambda: torch.empty(M, K, dtype=dtype, device=DEV).normal_(generator=gen)
    x, h, dn = big(), big(), big()
    g_post, g_pre = (torch.rand(K, generator=gen, device=DEV) + 0.5 for _ in range(2))
    gate = None if not T else torch.randn(-(-M // T), K, generator=gen, device=DEV).to(dtype)
    bs, tol = 0.5, (-(-M // 512) + 48) * 2.0 ** -24 + 2.0 ** -17
    _, _, dgate, dg_post, dg_pre = fn.flashnorm_block_residual_bwd(
        x, h, h, dn, g_post=g_post, eps_post=EPS_POST, gate=gate, rows_per_gate=T or 1, branch_scale=bs, g_pre=g_pre,
        eps_pre=EPS_PRE)
    cols = torch.tensor([0, 1, 7, 8, K // 2, K - 9, K - 1], device=DEV)
    sums = {n: torch.zeros(2, len(cols), dtype=torch.float64, device=DEV) for n in ("post", "pre")}  # values, magnitudes
    gates = torch.zeros(2, -(-M // T) if T else 0, len(cols), dtype=torch.float64, device=DEV)
    for m in range(0, M, 4096):
        rows = slice(m, min(M, m + 4096))
        at = torch.arange(m, rows.stop, device=DEV) // T if T else None
        X, D = x[rows].double(), dn[rows].double() * g_pre
        p = (EPS_POST + X.square().mean(1, keepdim=True)).rsqrt()
        z = X * p * g_post * bs
        H = h[rows].double()
        H = H + (z * gate[at].double() if T else z)
        r = (EPS_PRE + H.square().mean(1, keepdim=True)).rsqrt()
        t = r * (D * H).mean(1, keepdim=True)
        xp, H, D, dh, dnc = X[:, cols] * p, H[:, cols], D[:, cols], h[rows][:, cols].double(), dn[rows][:, cols].double()
        zc = z[:, cols]
        dH, mag = dh + r * (D - H * r * t), dh.abs() + r * (D.abs() + (H * r * t).abs())
        Hm = h[rows][:, cols].double().abs() + (zc * (gate[at][:, cols].double() if T else 1.0)).abs()
        gc = bs * (gate[at][:, cols].double() if T else 1.0)
        for name, v, a in (("post", dH * gc * xp, mag * abs(gc) * xp.abs()), ("pre", dnc * H * r, dnc.abs() * Hm * r)):
            sums[name] += torch.stack((v.sum(0), a.sum(0)))
        if T:
            gates[0].index_add_(0, at, dH * zc)
            gates[1].index_add_(0, at, mag * zc.abs())
    for name, got in (("post", dg_post), ("pre", dg_pre)):
        ref, mag = sums[name]
        over = (got[cols].double() - ref).abs() / (2.0 ** -24 * ref.abs() + tol * mag)
        assert torch.isfinite(got).all() and over.max() <= 1, (name, over.tolist())
    if T:
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        over = (dgate[:, cols].double() - gates[0]).abs() / (half * gates[0].abs() + tol * gates[1])
        assert torch.isfinite(dgate).all() and over.max() <= 1, float(over.max())
