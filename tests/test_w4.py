"""4-bit weights on the GPU: quantising, packing and reading back, and the products, against 64-bit
results computed on the CPU from the same codes.

Tolerances.  An output is rounded once to bf16: half a step, 2^-8 relative.  Before that:
  few rows    a group's sum runs in fp32 over terms a (128 + q), whose partial sums stay below 143 sum |a|, and
              (128 + z) sum a, below 191 sum |a|.  At most 16 roundings of such sums (4 matrix-core steps for
              each, two roundings a step), each at most 2^-23, are 16 * 334 * 2^-23 < 2^-10 of |s| sum |a|,
              i.e. 2^-13 of T = 8 sum |a s|;
  many rows   a weight (q - z) s is rounded to 11 bits, 2^-12 of it, after its scale, 2^-12 too, and so is a g
              where g is applied at run time: 1.5 * 2^-11 of A = sum |a w| together.  What fp16's subnormals
              lose lies 2^-39 (activations) and 2^-34 (weights) below the row's or column's largest value.
A call may go either way, so the tests allow 2^-13 T + 1.5 * 2^-11 A.  Over many outputs the error's root
mean square is what holds tighter: the output's rounding, a uniform error of at most half a step, 2^-8 /
sqrt(3) of the outputs', and beside it independent errors of 2^-12 / sqrt(3) per term, together within 2%.
"""
import numpy as np
import pytest
import torch

import __graft_entry__ as graft

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return flashnorm


def weights(K, N, group, zeros, seed):
    gen = torch.Generator().manual_seed(seed)
    groups = -(-K // group)
    codes = torch.randint(0, 16, (K, N), generator=gen, dtype=torch.uint8)
    scales = ((torch.rand(groups, N, generator=gen) + 0.5) * K ** -0.5 / 4).to(torch.bfloat16)
    z = torch.randint(0, 64, (groups, N), generator=gen, dtype=torch.uint8) if zeros == "wide" else \
        torch.randint(0, 16, (groups, N), generator=gen, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def dense(codes, scales, z, group):
    """The weight in 64 bits, and the magnitude 8 |s| of the tolerance."""
    K = codes.shape[0]
    s = scales.double().repeat_interleave(group, 0)[:K]
    zz = z.double().repeat_interleave(group, 0)[:K] if z is not None else torch.full_like(s, 8.0)
    return (codes.double() - zz) * s, 8.0 * s.abs()


def acts(M, K, seed):
    gen = torch.Generator().manual_seed(seed + 1000)
    a = torch.randn(M, K, generator=gen)
    a[::7] *= 20.0
    return a.to(torch.bfloat16)


def check(y, ref, tol, what):
    got = y.float().cpu().double()
    assert got.shape == ref.shape
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - tol
    assert over.max() <= 0, (what, float(over.max()), int((over > 0).sum()))
    if ref.numel() >= 4096:
        rms = ((got - ref).square().mean() / ref.square().mean()).sqrt()
        assert rms <= 1.02 * 2.0 ** -8 / 3 ** 0.5, (what, float(rms))


def linear_ref(a, W, T, g=None, scale=None):
    """The result in 64 bits and what it may be off by before its rounding."""
    x = a.double()
    s = (EPS + x.square().mean(1, keepdim=True)).rsqrt() if scale is None else scale
    if g is not None:
        x = x * g.double()
    return (x @ W) * s, 2.0 ** -13 * (x.abs() @ T) * s.abs() + 1.5 * 2.0 ** -11 * (x.abs() @ W.abs()) * s.abs()


SHAPES = [  # M, K, N: from one token to many, widths and depths that end inside a block or a group
    (1, 4096, 512), (1, 8, 1), (3, 40, 17), (5, 11008, 256), (7, 128, 16), (16, 72, 333), (16, 1000, 1376), (16, 2048, 6144),
    (17, 136, 40), (32, 512, 2064), (33, 256, 96), (64, 4096, 512), (100, 200, 333), (129, 1024, 272), (333, 520, 1000),
    (1000, 1160, 328), (2048, 256, 512)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_linear(fn, M, K, N, group):
    zeros = (False, True, "wide")[(M + K + group // 32) % 3]
    codes, scales, z = weights(K, N, group, zeros, M + K + N)
    a, (W, T) = acts(M, K, M), dense(codes, scales, z, group)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), None if z is None else z.to(DEV), group=group)
    inv = torch.full((M,), float("nan"), device=DEV)
    y = fn.flashnorm_linear_w4(a.to(DEV), w4, EPS, inv_rms=inv)
    ref, mag = linear_ref(a, W, T)
    check(y, ref, 2.0 ** -8 * ref.abs() + mag, (M, K, N, group, zeros))
    s = (EPS + a.double().square().mean(1)).rsqrt()
    assert ((inv.cpu().double() - s) / s).abs().max() < 1e-5


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(1, 4096, 128), (9, 520, 333), (16, 136, 2064), (40, 1024, 96), (200, 776, 520), (513, 256, 1040)])
def test_linear_run_time_g_and_bias(fn, M, K, N, group):
    codes, scales, z = weights(K, N, group, M % 2 == 0, M + N)
    a, (W, T) = acts(M, K, M), dense(codes, scales, z, group)
    gen = torch.Generator().manual_seed(M)
    g, bias = torch.randn(K, generator=gen) + 1.0, torch.randn(N, generator=gen)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), None if z is None else z.to(DEV), group=group)
    y = fn.flashnorm_linear_w4(a.to(DEV), w4, EPS, g=g.to(DEV), bias=bias.to(DEV))
    ref, mag = linear_ref(a, W, T, g)
    ref = ref + bias.double()
    check(y, ref, 2.0 ** -8 * ref.abs() + mag + 2.0 ** -23 * bias.abs(), (M, K, N, group))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,F,with_g", [(1, 4096, 256, False), (4, 72, 9, True), (16, 1000, 688, False), (13, 256, 5504, True),
                                          (50, 520, 200, True), (128, 1024, 344, False), (700, 264, 333, False), (1030, 512, 256, True)])
def test_glu(fn, M, K, F, with_g, group):
    codes, scales, z = weights(K, 2 * F, group, F % 2 == 1, M + F)
    a, (W, T) = acts(M, K, M), dense(codes, scales, z, group)
    g = torch.rand(K, generator=torch.Generator().manual_seed(F)) + 0.5 if with_g else None
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), None if z is None else z.to(DEV), layout=fn.FN_LAYOUT_GLU, group=group)
    y = fn.flashnorm_glu_w4(a.to(DEV), w4, EPS, g=None if g is None else g.to(DEV))
    t, mag = linear_ref(a, W, T, g)
    G, U, eG, eU = t[:, :F], t[:, F:], mag[:, :F], mag[:, F:]
    ref = G * torch.sigmoid(G) * U
    # |silu'| <= 1.1, |silu(t)| <= |t|; the fast exponential and quotient: 2^-20 relative
    tol = (2.0 ** -8 + 2.0 ** -20) * ref.abs() + 1.1 * eG * (U.abs() + eU) + G.abs() * eU
    check(y, ref, tol, (M, K, F, with_g, group))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N,scaled", [(1, 11008, 512, False), (6, 520, 4096, True), (16, 200, 77, True), (65, 1376, 256, False),
                                          (600, 392, 264, True)])
def test_rowscale(fn, M, K, N, scaled, group):
    codes, scales, z = weights(K, N, group, True, M + K)
    a, (W, T) = acts(M, K, M), dense(codes, scales, z, group)
    rs = torch.randn(M, generator=torch.Generator().manual_seed(K)) if scaled else None
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=group)
    y = fn.rowscale_linear_w4(a.to(DEV), w4, row_scale=None if rs is None else rs.to(DEV))
    ref, mag = linear_ref(a, W, T, scale=torch.ones(M, 1, dtype=torch.float64) if rs is None else rs.double()[:, None])
    check(y, ref, 2.0 ** -8 * ref.abs() + mag, (M, K, N, scaled, group))


def quantise(W, g, group, zero_points):
    """The definition in 64 bits (numpy): codes, scales, zero points and the weight."""
    w = W.double().numpy() * (g.double().numpy()[:, None] if g is not None else 1.0)
    K, N = w.shape
    out = np.empty((K, N))
    for k in range(0, K, group):
        v = w[k:k + group]
        lo, hi = np.minimum(v.min(0), 0.0), np.maximum(v.max(0), 0.0)
        s = (hi - lo) / 15.0 if zero_points else np.maximum(hi, -lo) / 7.0
        m, e = np.frexp(s)
        s = np.ldexp(np.rint(m * 4096.0), e - 12)
        s[s < 2.0 ** -126] = 0.0
        with np.errstate(divide="ignore", invalid="ignore"):
            z = np.clip(np.rint(-lo / s), 0, 15) if zero_points else np.full(N, 8.0)
            z = np.where(s > 0, z, 8.0)
            q = np.where(s > 0, np.clip(np.rint(v / s) + z, 0, 15), z)
        out[k:k + group] = (q - z) * s
    return out


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zero_points", [False, True])
@pytest.mark.parametrize("K,N,dtype,view,glu", [
    (8, 1, torch.bfloat16, "rows", False), (40, 17, torch.float32, "rows", False), (72, 34, torch.bfloat16, "t", True),
    (130, 48, torch.float32, "t", False), (576, 1536, torch.bfloat16, "t", False), (1000, 86, torch.float32, "third", True),
    (512, 333, torch.bfloat16, "offset", False)])
def test_fold_is_the_definition_exactly(fn, K, N, dtype, view, glu, zero_points, group):
    gen = torch.Generator().manual_seed(K + N)
    W = torch.randn(K, N, generator=gen) * torch.exp(2 * torch.randn(K, 1, generator=gen))
    W[: K // 2, N // 2] = 0.0                              # a group of zeros
    W[:, 0] = torch.arange(K).float() % 15 - 7.0           # quotients that are whole
    if N > 3:
        W[:, 3] = (torch.arange(K).float() % 29) / 2 - 7.0  # and halves: ties
        W[:, 2] = W[:, 2].abs() + 1.0                       # one sign
    W = W.to(dtype)
    g = None if (K + group) % 3 == 0 else (torch.rand(K, generator=gen) * 2 - 0.5)
    if view == "t":
        Wd = W.t().contiguous().to(DEV).t()
    elif view == "third":
        Wd = torch.zeros(K, 3 * N, dtype=dtype, device=DEV)[:, 1::3]
        Wd.copy_(W)
    elif view == "offset":
        Wd = torch.zeros(K + 1, N + 5, dtype=dtype, device=DEV)[1:, 5:]
        Wd.copy_(W)
    else:
        Wd = W.to(DEV)
    w4 = fn.fold_weights_w4(Wd, None if g is None else g.to(DEV), layout=fn.FN_LAYOUT_GLU if glu else fn.FN_LAYOUT_LINEAR,
                            group=group, zero_points=zero_points)
    got = fn.unpack_weights_w4(w4).cpu().double().numpy()
    ref = quantise(W, g, group, zero_points)
    assert np.array_equal(got, ref), (np.abs(got - ref).max(), int((got != ref).sum()))


def test_fold_values_that_have_no_scale(fn):
    W = torch.ones(256, 6, dtype=torch.float32)
    W[3, 1] = float("nan")
    W[130, 2] = float("inf")
    W[:, 3] = 1e-40           # a scale below 2^-126: zeros
    W[:, 4] = 3e38
    g = torch.full((256,), 100.0)  # column 4 leaves fp32
    w4 = fn.fold_weights_w4(W.to(DEV), g.to(DEV), group=128)
    got = fn.unpack_weights_w4(w4).cpu()
    bad = torch.zeros(256, 6, dtype=torch.bool)
    bad[:128, 1] = bad[128:, 2] = bad[:, 4] = True
    assert torch.equal(torch.isnan(got), bad)
    assert (got[:, 3] == 0).all()
    y = fn.flashnorm_linear_w4(torch.ones(3, 256, dtype=torch.bfloat16, device=DEV), w4, EPS).float().cpu()
    assert torch.equal(torch.isnan(y), torch.tensor([[False, True, True, False, True, False]] * 3))


@pytest.mark.parametrize("scale_dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K,N,group,glu", [(8, 2, 32, True), (200, 66, 64, False), (257, 20, 128, True), (384, 333, 32, False)])
def test_pack_and_unpack(fn, K, N, group, glu, scale_dtype):
    codes, scales, z = weights(K, N, group, "wide", K)
    scales = (scales.float() * (1 + 2.0 ** -9)).to(scale_dtype)
    wide = torch.zeros(K, N + 3, dtype=torch.uint8, device=DEV)
    wide[:, 2:N + 2] = codes.to(DEV)
    w4 = fn.pack_weights_w4(wide[:, 2:N + 2], scales.to(DEV), z.to(DEV), group=group,
                            layout=fn.FN_LAYOUT_GLU if glu else fn.FN_LAYOUT_LINEAR)
    s = scales.float()
    if scale_dtype == torch.float32:  # 12 significant bits
        m, e = np.frexp(s.numpy())
        s = torch.from_numpy(np.ldexp(np.rint(m * 4096), e - 12).astype(np.float32))
    ref, _ = dense(codes, s, z, group)
    assert torch.equal(fn.unpack_weights_w4(w4).cpu().double(), ref)


def test_fold_then_product_is_near_the_full_weight(fn):
    """The whole path: quantising costs half a step of the scale at most."""
    K, N, M = 512, 320, 24
    gen = torch.Generator().manual_seed(5)
    W, g = torch.randn(N, K, generator=gen).to(torch.bfloat16), torch.rand(K, generator=gen) + 0.5
    a = acts(M, K, 1)
    w4 = fn.fold_weights_w4(W.to(DEV).t(), g.to(DEV), group=64, zero_points=True)
    y = fn.flashnorm_linear_w4(a.to(DEV), w4, EPS).float().cpu().double()
    held = torch.from_numpy(quantise(W.t(), g, 64, True))
    ref = (a.double() @ held) * (EPS + a.double().square().mean(1, keepdim=True)).rsqrt()
    full = (a.double() @ (W.double().t() * g.double()[:, None])) * (EPS + a.double().square().mean(1, keepdim=True)).rsqrt()
    assert ((y - ref).norm() / ref.norm()) <= 2.0 ** -8
    step = (held - W.double().t() * g.double()[:, None]).abs().max() * 2
    assert ((ref - full).norm() / full.norm()) <= float(step) / 2 / float((W.double().t() * g.double()[:, None]).square().mean().sqrt())


@pytest.mark.parametrize("M", [1, 4, 16, 40, 300])
def test_rows_that_hold_nan_or_inf_stay_alone(fn, M):
    K, N = 264, 100
    codes, scales, z = weights(K, N, 64, True, 3)
    a = acts(M, K, 2)
    bad = sorted({0, M // 2, M - 1})
    clean = a.clone()
    for i, r in enumerate(bad):
        a[r, (37 * i + 5) % K] = (float("nan"), float("inf"), float("-inf"))[i]
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=64)
    y, y0 = (fn.flashnorm_linear_w4(t.to(DEV), w4, EPS).cpu() for t in (a, clean))
    assert torch.isnan(y[bad]).all()
    keep = [r for r in range(M) if r not in bad]
    assert torch.equal(y[keep], y0[keep])


@pytest.mark.parametrize("M", [1, 16, 64, 200])
def test_zero_rows_and_zero_eps(fn, M):
    codes, scales, z = weights(128, 48, 32, True, 4)
    a = acts(M, 128, 6)
    a[0] = 0.0
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=32)
    assert (fn.flashnorm_linear_w4(a.to(DEV), w4, EPS)[0] == 0).all()
    y = fn.flashnorm_linear_w4(a.to(DEV), w4, 0.0)
    assert torch.isnan(y[0]).all() and torch.isfinite(y[1:]).all()


@pytest.mark.parametrize("M,K,N", [(2, 136, 40), (16, 1000, 333), (70, 520, 264), (300, 264, 1000)])
def test_views_and_what_lies_beside_them(fn, M, K, N):
    """Inputs inside wider rows whose padding is NaN; the output's padding and neighbours stay as they were."""
    codes, scales, z = weights(K, N, 128, False, 8)
    a, (W, T) = acts(M, K, 3), dense(codes, scales, z, 128)
    wide = torch.full((M + 2, K + 24), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[1:-1, 8:K + 8] = a.to(DEV)
    out = torch.full((M + 2, (N + 7) // 8 * 8 + 16), 3.0, dtype=torch.bfloat16, device=DEV)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), group=128)
    fn.flashnorm_linear_w4(wide[1:-1, 8:K + 8], w4, EPS, out=out[1:-1, 8:N + 8])
    ref, mag = linear_ref(a, W, T)
    check(out[1:-1, 8:N + 8], ref, 2.0 ** -8 * ref.abs() + mag, (M, K, N))
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[1:-1, 8:N + 8] = False
    assert (out[keep] == 3.0).all()


@pytest.mark.parametrize("M", [0, 1, 16, 40, 300])
def test_repeats_graph_and_stream(fn, M):
    """The same bits on a repeat, on another stream, and in every replay of a captured graph."""
    K, F = 520, 200
    codes, scales, z = weights(K, 2 * F, 32, True, 9)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), layout=fn.FN_LAYOUT_GLU, group=32)
    a, g = acts(M, K, 4).to(DEV), torch.rand(K, device=DEV) + 0.5
    y = fn.flashnorm_glu_w4(a, w4, EPS, g=g)
    assert y.shape == (M, F)
    assert torch.equal(fn.flashnorm_glu_w4(a, w4, EPS, g=g), y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = fn.flashnorm_glu_w4(a, w4, EPS, g=g, stream=side)
    y3 = fn.flashnorm_glu_w4(a, w4, EPS, g=g, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y2, y) and torch.equal(y3, y)
    if M == 0:
        return
    graph = torch.cuda.CUDAGraph()
    ain = a.clone()
    with torch.cuda.graph(graph):
        yg = fn.flashnorm_glu_w4(ain, w4, EPS, g=g)
    for i in range(3):
        ain.copy_(acts(M, K, 20 + i).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(yg, fn.flashnorm_glu_w4(ain, w4, EPS, g=g)), i


def test_a_feed_forward_block(fn):
    """Fold, GLU, down projection and block residual in a row, as a decoder layer runs them, at one
    token and at many: against 64 bits from the held weights, step by step."""
    K, F, H = 512, 1376, 512
    gen = torch.Generator().manual_seed(1)
    Wgu = (torch.randn(2 * F, K, generator=gen) * K ** -0.5).to(torch.bfloat16)
    Wd = (torch.randn(H, F, generator=gen) * F ** -0.5).to(torch.bfloat16)
    g_in, g_post = torch.rand(K, generator=gen) + 0.5, torch.rand(H, generator=gen) + 0.5
    up = fn.fold_weights_w4(Wgu.to(DEV).t(), g_in.to(DEV), layout=fn.FN_LAYOUT_GLU, group=64, zero_points=True)
    down = fn.fold_weights_w4(Wd.to(DEV).t(), group=32)
    Wu64, Wd64 = (fn.unpack_weights_w4(w).cpu().double() for w in (up, down))
    for M in (1, 16, 75, 260):
        h = acts(M, K, M)
        hd = h.to(DEV)
        f = fn.flashnorm_glu_w4(hd, up, EPS)
        x = fn.rowscale_linear_w4(f, down)
        fn.flashnorm_block_residual(x, hd, g_post=g_post.to(DEV), eps_post=EPS, branch_scale=0.5, out=hd)
        hr = h.double()
        t = (hr @ Wu64) * (EPS + hr.square().mean(1, keepdim=True)).rsqrt()
        fr = t[:, :F] * torch.sigmoid(t[:, :F]) * t[:, F:]
        xr = fr @ Wd64
        out = hr + 0.5 * xr * (EPS + xr.square().mean(1, keepdim=True)).rsqrt() * g_post.double()
        # three roundings to bf16 on the way, each at most 2^-8 of its row
        err = (hd.float().cpu().double() - out).norm(dim=1) / out.norm(dim=1)
        assert err.max() <= 3 * 2.0 ** -8, (M, float(err.max()))


def test_workspace(fn):
    """A caller's workspace, one for several calls; what lies behind it stays as it was."""
    K, N = 512, 4000
    codes, scales, z = weights(K, N, 64, True, 11)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=64)
    need = {M: fn.lib().flashnorm_w4_workspace_size(M, K, N, 0, 64) for M in (1, 16, 300, 2000)}
    assert need[1] == need[16] == 0 and need[2000] > 2000 * K * 2
    ws = torch.full((max(need.values()) + 64,), 7, dtype=torch.uint8, device=DEV)
    for M in (2000, 300, 1, 2000):
        a = acts(M, K, M).to(DEV)
        y = fn.flashnorm_linear_w4(a, w4, EPS, workspace=ws)
        assert torch.equal(y, fn.flashnorm_linear_w4(a, w4, EPS))
    assert (ws[max(need.values()):] == 7).all()
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a, w4, EPS, workspace=ws[:need[2000] - 1])
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a, w4, EPS, workspace=ws.cpu())


@pytest.mark.parametrize("M", [3, 200])
def test_ranges_of_scales_and_activations(fn, M):
    """Scales across a column and values across a row that lie far apart, and far from one."""
    K, N = 512, 64
    codes, scales, z = weights(K, N, 32, True, 12)
    scales = scales.float() * torch.exp2(torch.randint(-20, 1, scales.shape, generator=torch.Generator().manual_seed(1)).float())
    scales[:, 1] *= 2.0 ** 100
    scales[:, 2] *= 2.0 ** -90
    scales[:, 3] = 0.0
    scales[::2, 4] = 0.0
    a = acts(M, K, 9).float() * torch.exp2(torch.randint(-12, 13, (M, K), generator=torch.Generator().manual_seed(2)).float())
    a[1] *= 2.0 ** 50
    a[2] *= 2.0 ** -40
    a = a.to(torch.bfloat16)
    scales = scales.to(torch.bfloat16)
    W, T = dense(codes, scales, z, 32)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=32)
    rs = torch.ones(M)
    y = fn.rowscale_linear_w4(a.to(DEV), w4, row_scale=rs.to(DEV))
    ref, mag = linear_ref(a, W, T, scale=rs.double()[:, None])
    # 2^50 times 2^100 and a weight of 2^-5: beyond bf16 (2^128), so infinite or NaN and no number
    held = ref.abs() < 2.0 ** 127
    assert held.sum() == held.numel() - 1 and not torch.isfinite(y[1, 1])
    y[1, 1], ref[1, 1] = 0.0, 0.0
    check(y, ref, 2.0 ** -8 * ref.abs() + mag, M)


def test_refusals_of_the_binding(fn):
    codes, scales, z = weights(64, 32, 32, True, 1)
    w4 = fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=32)
    a = acts(4, 64, 1).to(DEV)
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(acts(4, 72, 1).to(DEV), w4, EPS)          # another K
    with pytest.raises(ValueError):
        fn.flashnorm_glu_w4(a, w4, EPS)                                    # another layout
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a.cpu(), w4, EPS)
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a, w4, EPS, g=torch.ones(64))               # g on the host
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a, w4, EPS, out=torch.empty(4, 40, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a, w4, EPS, out=torch.empty(4, 32, device=DEV))
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a, w4, EPS, inv_rms=torch.empty(3, device=DEV))
    with pytest.raises(ValueError):
        fn.flashnorm_linear_w4(a.t(), w4, EPS)
    for call in (lambda: fn.flashnorm_linear_w4(a.float(), w4, EPS),       # fp32 activations
                 lambda: fn.flashnorm_linear_w4(a, w4, -1.0),
                 lambda: fn.rowscale_linear_w4(a, w4, out=a[:, :32])):      # the output over the input
        with pytest.raises(fn.FlashNormError):
            call()
    with pytest.raises(TypeError):
        fn.flashnorm_linear_w4(a.half(), w4, EPS)
    with pytest.raises(ValueError):
        fn.pack_weights_w4(codes.to(DEV), scales.to(DEV)[:1], z.to(DEV), group=32)
    with pytest.raises(ValueError):
        fn.pack_weights_w4(codes.to(DEV), scales.to(DEV), z.to(DEV), group=48)
    with pytest.raises(ValueError):
        fn.pack_weights_w4(codes.to(DEV).int(), scales.to(DEV), z.to(DEV), group=32)
    with pytest.raises(ValueError):
        fn.fold_weights_w4(torch.ones(8, 7, device=DEV), layout=fn.FN_LAYOUT_GLU)
    with pytest.raises(ValueError):
        fn.W4Weight(w4.data[:-1], 64, 32, fn.FN_LAYOUT_LINEAR, 32)


def test_refusals_of_the_fold(fn):
    W = torch.ones(64, 32, device=DEV)
    g = torch.ones(64, device=DEV)
    for bad in (dict(g=g.cpu()), dict(g=g[:63]), dict(g=g.double()), dict(group=48), dict(group=(1 << 32) + 32), dict(layout=2),
                dict(layout=1 << 32)):
        with pytest.raises(ValueError):
            fn.fold_weights_w4(W, **bad)
    for W2 in (W[0], W.cpu(), W[:0], W[None]):
        with pytest.raises(ValueError):
            fn.fold_weights_w4(W2)
    with pytest.raises(TypeError):
        fn.fold_weights_w4(W.half())
    with pytest.raises(TypeError):
        fn.fold_weights_w4(W, group="32")
    w4 = fn.fold_weights_w4(W, zero_points=np.bool_(True), group=32)
    assert (w4.K, w4.N, w4.layout, w4.group) == (64, 32, fn.FN_LAYOUT_LINEAR, 32)
    assert np.array_equal(fn.unpack_weights_w4(w4).cpu().numpy(), quantise(W.cpu(), None, 32, True))
    w4.group = 64  # a smaller scale table, but another one
    w4.K = 1 << 16
    with pytest.raises(ValueError):
        fn.unpack_weights_w4(w4)


def test_fold_on_another_stream(fn):
    W, g = torch.randn(520, 96, device=DEV), torch.rand(520, device=DEV) + 0.5
    ref = fn.unpack_weights_w4(fn.fold_weights_w4(W, g, group=32, zero_points=True))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w4 = fn.fold_weights_w4(W, g, group=32, zero_points=True, stream=side)
    got = fn.unpack_weights_w4(w4, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, ref)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K,N,rows,glu", [(8, 1, True, False), (300, 75, True, False), (512, 190, False, True), (600, 74, True, True),
                                          (1024, 66, True, False), (1032, 40, True, False), (2048, 33, False, False),
                                          (2049, 34, False, True), (4100, 70, True, True)])
def test_columns_norms(fn, K, N, rows, glu, group):
    """The power of two behind each packed column of a fold: its largest scale lies in [2^9, 2^10) times it, one for
    columns without a finite scale (padding, zeros, NaN)."""
    gen = torch.Generator().manual_seed(K + N)
    W = torch.randn(K, N, generator=gen) * torch.exp2(torch.randint(-40, 40, (1, N), generator=gen).float())
    if N > 3:
        W[:, 1] = 0.0
        W[K // 2, 2] = float("nan")
    W = W if rows else W.t().contiguous().t()
    w4 = fn.fold_weights_w4(W.to(DEV), layout=fn.FN_LAYOUT_GLU if glu else fn.FN_LAYOUT_LINEAR, group=group)
    NP = 2 * (-(-(N // 2) // 16) * 16) if glu else -(-N // 16) * 16
    groups = -(-K // 128) * (128 // group)
    tail = w4.data.cpu()[-4 * NP * (groups + 1):]
    words, norms = tail[:4 * NP * groups].view(torch.int32).view(groups, NP), tail[4 * NP * groups:].view(torch.float32).numpy()
    top = (words & 0x7ffff000).view(torch.float32).abs().numpy()
    bad = ~np.isfinite(top).all(0) | (top.max(0) == 0)
    assert (norms[bad] == 1.0).all() and bad.sum() >= (2 if N > 3 else 0)
    e = np.frexp(top.max(0)[~bad])[1]
    assert np.array_equal(norms[~bad], np.ldexp(1.0, 10 - e).astype(np.float32))


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("K,N,lead,glu", [(8, 1, 3, False), (130, 17, 1, False), (1024, 46, 0, True), (1025, 46, 5, True),
                                          (1400, 130, 0, False), (300, 64, 7, False)])
def test_fold_of_rows_at_any_offset(fn, K, N, lead, glu, group):
    """bf16 weights in rows (unit column stride) that start at any element, amid NaN that must not be read into a
    group: exactly the definition."""
    gen = torch.Generator().manual_seed(K * N)
    W = torch.randn(K, N, generator=gen).to(torch.bfloat16)
    wide = torch.full((K + 1, N + lead + 3), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:K, lead:N + lead] = W.to(DEV)
    g = torch.rand(K, generator=gen) + 0.5
    w4 = fn.fold_weights_w4(wide[:K, lead:N + lead], g.to(DEV), layout=fn.FN_LAYOUT_GLU if glu else fn.FN_LAYOUT_LINEAR,
                            group=group, zero_points=True)
    assert np.array_equal(fn.unpack_weights_w4(w4).cpu().double().numpy(), quantise(W, g, group, True))
