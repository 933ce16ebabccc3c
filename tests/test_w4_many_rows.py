"""4-bit products of more rows than one launch takes: they go in pieces, in one workspace.  Tolerances of test_w4.py."""
import pytest
import torch

import __graft_entry__ as graft
from test_w4 import EPS
from test_w4_shapes import make, plan, ref_of

DEV = "cuda:0"
M = (1 << 22) + 37


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    if torch.cuda.mem_get_info()[0] < 32 << 30:
        pytest.skip("needs 32 GB of free GPU memory")
    return flashnorm


def near(y, ref, tol, what):
    over = (y.double() - ref).abs() - tol
    assert torch.isfinite(y).all() and over.max() <= 0, (what, float(over.max()), int((over > 0).sum()))


@pytest.mark.gpu
@pytest.mark.parametrize("N", [16, 41])
def test_linear_and_row_scale(fn, N):
    K, G = 16, 32
    p = plan(M, K, N, False, G, False)
    assert p.many  # the pass over the rows is the launch that cannot take them
    a, w4, W, T = make(fn, M, K, N, False, G, 1)
    inv = torch.full((M,), float("nan"), device=DEV)
    y = fn.flashnorm_linear_w4(a, w4, EPS, inv_rms=inv)
    ref, mag = ref_of(a, W, T)
    near(y, ref, 2.0 ** -8 * ref.abs() + mag, "linear")
    s = (EPS + a.double().square().mean(1)).rsqrt()
    assert ((inv.double() - s) / s).abs().max() < 1e-5
    scale = torch.randn(M, device=DEV)
    y = fn.rowscale_linear_w4(a, w4, row_scale=scale)
    ref, mag = ref_of(a, W, T, scale=scale)
    near(y, ref, 2.0 ** -8 * ref.abs() + mag, "row scale")
    rows = slice(M - 45, M)  # the last piece begins there
    assert torch.equal(y[rows], fn.rowscale_linear_w4(a, w4, row_scale=scale)[rows])


@pytest.mark.gpu
def test_glu_in_a_workspace_of_one_piece(fn):
    K, F, G = 8, 24, 64
    a, w4, W, T = make(fn, M, K, 2 * F, True, G, 2)
    size = fn.lib().flashnorm_w4_workspace_size
    need = size(M, K, 2 * F, 1, G)
    assert 0 < need <= size((1 << 22) - 1, K, 2 * F, 1, G)  # the pieces share it
    ws = torch.full((need + 64,), 7, dtype=torch.uint8, device=DEV)
    y = fn.flashnorm_glu_w4(a, w4, EPS, workspace=ws)
    assert (ws[need:] == 7).all()
    t, mag = ref_of(a, W, T)
    g, u, eg, eu = t[:, :F], t[:, F:], mag[:, :F], mag[:, F:]
    ref = g * torch.sigmoid(g) * u
    near(y, ref, (2.0 ** -8 + 2.0 ** -20) * ref.abs() + 1.1 * eg * (u.abs() + eu) + g.abs() * eu, "GLU")


def test_outputs_that_no_card_holds():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    lib, N = flashnorm.lib(), 1 << 20
    need = lib.flashnorm_w4_workspace_size(1 << 30, 8, N, 0, 32)
    assert lib.flashnorm_linear_w4(0x100000, 1 << 30, 8, 8, 1, 0, 0x10000000, N, 32, 1e-6, 0, 1 << 60, N, 1, 0, 1 << 61, need,
                                   None) == -9
