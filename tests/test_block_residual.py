"""The block residual and its gradients on the GPU, against 64 bits on the CPU (the gradients by
automatic differentiation of the definition, and by differences).

Tolerances.  An output is rounded once: half a step of its type, relative.  What it is rounded from
carries fp32 errors: a few roundings per element, and the row sums, in which a value passes at most 32
additions in a thread and 10 more across threads (44 roundings of 2^-24 with the products' own, below
2^-18).  So an element is off by at most 2^-18 of the sum of its terms' magnitudes, taken for the row
sums as the sums of magnitudes; the tests allow 2^-17.  Sums over rows pass at most M / 1024 + 1
additions in a unit (8 at the sizes here), 64 + 16 across units: 2^-17 of the sum of magnitudes, twice
that with the terms' own errors."""
import pytest
import torch

import __graft_entry__ as graft

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -17
EPS_POST, EPS_PRE = 1e-5, 1e-6


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return flashnorm


def make(M, K, dtype, post, T, pre, seed=0):
    gen = torch.Generator().manual_seed(seed + M * 31 + K)
    rnd = lambda *s: torch.randn(*s, generator=gen)
    x = {"x": (rnd(M, K) * 3 * torch.exp(rnd(M, 1))).to(dtype), "h": rnd(M, K).to(dtype), "dh_out": rnd(M, K).to(dtype)}
    if post:
        x["g_post"] = rnd(K) * 0.3 + 1.0
    if T:
        x["gate"] = rnd(-(-M // T), K).to(dtype)
    if pre:
        x["g_pre"] = rnd(K) * 0.3 + 1.0
        x["dn"] = rnd(M, K).to(dtype)
    return x


def gate_of(v, M, T):
    return v["gate"].double()[torch.arange(M) // T] if "gate" in v else 1.0


def terms(v, T, rs, bs):
    """The forward pass in 64 bits, with the magnitudes of out's terms."""
    d = {k: t.double() for k, t in v.items()}
    M = d["x"].shape[0]
    p = (EPS_POST + d["x"].square().mean(1, keepdim=True)).rsqrt() if "g_post" in v else torch.ones(M, 1, dtype=torch.float64)
    gp = d["g_post"] if "g_post" in v else 1.0
    z = d["x"] * p * gp
    gate = gate_of(v, M, T)
    out = rs * d["h"] + bs * gate * z
    mag = (rs * d["h"]).abs() + (bs * gate * z).abs()
    r = (EPS_PRE + out.square().mean(1, keepdim=True)).rsqrt()
    return d, p, gp, z, gate, out, mag, r


def close(got, ref, tol, what):
    got = got.double().cpu()
    assert got.shape == ref.shape
    over = (got - ref).abs() - tol
    assert torch.isfinite(got).all() and over.max() <= 0, (what, float(over.max()), int((over > 0).sum()))


def kwargs(v, T, rs, bs):
    to = lambda n: v[n].to(DEV) if n in v else None
    return dict(g_post=to("g_post"), eps_post=EPS_POST, gate=to("gate"), rows_per_gate=T or 1, res_scale=rs, branch_scale=bs,
                g_pre=to("g_pre"), eps_pre=EPS_PRE)


CASES = [  # M, K, rows per gate (0: none), post-norm, next norm
    (1, 8, 0, True, True), (1, 4096, 0, True, False), (3, 40, 1, False, True), (5, 512, 2, True, True), (7, 520, 7, True, True),
    (2, 1024, 1, True, True), (9, 1032, 4, False, False), (4, 2048, 0, True, True), (3, 4104, 2, True, True),
    (2, 8192, 1, True, True), (2, 16384, 2, True, True), (3, 12296, 1, True, True), (1999, 576, 0, True, True), (1500, 264, 1, True, True),
    (2500, 72, 3, True, True), (1300, 136, 1300, True, True), (1100, 200, 333, True, True), (4100, 64, 2000, False, True),
    (2100, 8, 2, True, True)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,T,post,pre", CASES)
def test_forward(fn, M, K, T, post, pre, dtype):
    v = make(M, K, dtype, post, T, pre)
    rs, bs = (1.0, 0.5) if M % 2 else (0.75, -1.25)
    inv = torch.full((M,), float("nan"), device=DEV)
    out, normed = fn.flashnorm_block_residual(v["x"].to(DEV), v["h"].to(DEV), inv_rms=inv, **kwargs(v, T, rs, bs))
    d, p, gp, z, gate, ref, mag, r = terms(v, T, rs, bs)
    half = HALF[dtype]
    close(out, ref, half * ref.abs() + U * mag, "out")
    # the row's sum of squares has a relative error below that of its largest terms
    srel = U * (1 + (mag * ref.abs()).sum(1, keepdim=True) / (ref.square().sum(1, keepdim=True) + 1e-300))
    close(inv[:, None], r, r * srel, "inv_rms")
    if pre:
        n = ref * r * d["g_pre"]
        close(normed, n, half * n.abs() + (U * mag * r + srel * (ref * r).abs()) * d["g_pre"].abs() * (1 + half), "normed")
    else:
        assert normed is None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,T,post,pre", CASES)
def test_gradients(fn, M, K, T, post, pre, dtype):
    v = make(M, K, dtype, post, T, pre, seed=1)
    rs, bs = (1.0, 0.5) if M % 2 else (0.75, -1.25)
    with_dh = not (pre and M % 3 == 0)
    args = [v["x"].to(DEV), v["h"].to(DEV), v["dh_out"].to(DEV) if with_dh else None, v["dn"].to(DEV) if pre else None]
    got = dict(zip(("x", "h", "gate", "g_post", "g_pre"), fn.flashnorm_block_residual_bwd(*args, **kwargs(v, T, rs, bs))))
    # the definition, differentiated
    leaves = {n: v[n].double().requires_grad_(True) for n in ("x", "h", "gate", "g_post", "g_pre") if n in v}
    x = leaves["x"]
    z = x / (EPS_POST + x.square().mean(1, keepdim=True)).sqrt() * leaves["g_post"] if post else x
    if T:
        z = z * leaves["gate"][torch.arange(M) // T]
    o = rs * leaves["h"] + bs * z
    total = (o * v["dh_out"].double()).sum() if with_dh else 0.0
    if pre:
        n = o / (EPS_PRE + o.square().mean(1, keepdim=True)).sqrt() * leaves["g_pre"]
        total = total + (n * v["dn"].double()).sum()
    ref = dict(zip(leaves, torch.autograd.grad(total, list(leaves.values()))))
    # magnitudes of the terms
    d, p, gp, zz, gate, H, mag, r = terms(v, T, rs, bs)
    dho = d["dh_out"].abs() if with_dh else torch.zeros_like(H)
    D = dho.clone()
    if pre:
        a = (d["dn"] * d["g_pre"]).abs()
        Hn = mag * r
        D = D + r * (a + Hn * (a * Hn).mean(1, keepdim=True))
        # r itself is off by the relative error of a sum of squares
        D = D * (1 + (mag * H.abs()).sum(1, keepdim=True) / H.square().sum(1, keepdim=True).clamp_min(1e-300))
    bg = abs(bs) * (gate.abs() if T else torch.ones_like(H))
    xp = d["x"].abs() * p
    dz = bg * D
    half = HALF[dtype]
    tol = {"h": half * ref["h"].abs() + U * abs(rs) * D}
    if post:
        gpa = d["g_post"].abs()
        tol["x"] = half * ref["x"].abs() + U * p * (dz * gpa + xp * (dz * gpa * xp).mean(1, keepdim=True))
        tol["g_post"] = 2 * U * (dz * xp).sum(0)
    else:
        tol["x"] = half * ref["x"].abs() + U * dz
    if T:
        s = torch.zeros_like(ref["gate"]).index_add_(0, torch.arange(M) // T, abs(bs) * D * zz.abs())
        tol["gate"] = half * ref["gate"].abs() + 2 * U * s
    if pre:
        tol["g_pre"] = 2 * U * (d["dn"].abs() * mag * r).sum(0) * 2
    for name in ("x", "h", "gate", "g_post", "g_pre"):
        if name in ref:
            close(got[name], ref[name], tol[name], name)
        else:
            assert got[name] is None, name


def test_gradients_against_differences(fn):
    M, K, T, rs, bs = 6, 64, 3, 0.9, 1.3
    v = make(M, K, torch.float32, True, T, True, seed=2)
    got = fn.flashnorm_block_residual_bwd(v["x"].to(DEV), v["h"].to(DEV), v["dh_out"].to(DEV), v["dn"].to(DEV),
                                          **kwargs(v, T, rs, bs))

    def value(w):
        d, p, gp, z, gate, out, mag, r = terms(w, T, rs, bs)
        return float((out * d["dh_out"]).sum() + (out * r * d["g_pre"] * d["dn"]).sum())

    gen = torch.Generator().manual_seed(3)
    for name, g in zip(("x", "h", "gate", "g_post", "g_pre"), got):
        direction = torch.randn(v[name].shape, generator=gen, dtype=torch.float64)
        step = 1e-5
        up = value({**v, name: v[name].double() + step * direction})
        down = value({**v, name: v[name].double() - step * direction})
        slope = float((g.double().cpu() * direction).sum())
        # differences: step^2 and 2^-52 of the value over the step; the kernel's own error in fp32
        assert abs(slope - (up - down) / (2 * step)) <= 1e-5 * float(g.double().cpu().norm() * direction.norm()), name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K", [(1, 4096), (5, 264), (300, 1032)])
def test_in_place_and_views(fn, M, K, dtype):
    """out over h, normed over x, and rows inside wider ones whose padding is NaN."""
    v = make(M, K, dtype, True, 1, True, seed=4)
    kw = kwargs(v, 1, 1.0, 0.5)
    out, normed = fn.flashnorm_block_residual(v["x"].to(DEV), v["h"].to(DEV), **kw)
    x, h = v["x"].to(DEV), v["h"].to(DEV)
    o2, n2 = fn.flashnorm_block_residual(x, h, out=h, normed=x, **kw)
    assert o2 is h and n2 is x and torch.equal(h, out) and torch.equal(x, normed)
    pad = 8
    wide = lambda t: torch.nn.functional.pad(t.to(DEV), (pad, 3 * pad, 1, 1), value=float("nan"))[1:-1, pad:K + pad]
    kw["gate"] = wide(v["gate"])
    dst = [torch.full((M + 2, K + 4 * pad), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
    fn.flashnorm_block_residual(wide(v["x"]), wide(v["h"]), out=dst[0][1:-1, pad:K + pad], normed=dst[1][1:-1, pad:K + pad], **kw)
    for t, ref in zip(dst, (out, normed)):
        assert torch.equal(t[1:-1, pad:K + pad], ref)
        t[1:-1, pad:K + pad] = 7.0
        assert (t == 7.0).all()
    plain = fn.flashnorm_block_residual_bwd(v["x"].to(DEV), v["h"].to(DEV), v["dh_out"].to(DEV), v["dn"].to(DEV),
                                            **kwargs(v, 1, 1.0, 0.5))
    strided = fn.flashnorm_block_residual_bwd(wide(v["x"]), wide(v["h"]), wide(v["dh_out"]), wide(v["dn"]), **kw)
    for a, b in zip(plain, strided):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_row_stays_alone(fn, bad):
    M, K = 70, 520
    v = make(M, K, torch.bfloat16, True, 0, True, seed=5)
    kw = kwargs(v, 0, 1.0, 1.0)
    clean = fn.flashnorm_block_residual(v["x"].to(DEV), v["h"].to(DEV), **kw)
    v["x"][13, 7] = bad
    got = fn.flashnorm_block_residual(v["x"].to(DEV), v["h"].to(DEV), **kw)
    grads = fn.flashnorm_block_residual_bwd(v["x"].to(DEV), v["h"].to(DEV), v["dh_out"].to(DEV), v["dn"].to(DEV), **kw)
    rows = [i for i in range(M) if i != 13]
    for a, b in zip(got, clean):
        assert torch.equal(a[rows], b[rows])
    assert torch.isnan(got[1][13]).any()
    assert torch.isfinite(grads[0][rows]).all() and torch.isfinite(grads[1][rows]).all() and torch.isnan(grads[0][13]).any()


def test_zero_rows(fn):
    """A row of zeros: zeros with an epsilon, NaN as the formula gives it without."""
    z = torch.zeros(3, 64, device=DEV)
    one = torch.ones(64, device=DEV)
    out, n = fn.flashnorm_block_residual(z, z, g_post=one, eps_post=1e-6, g_pre=one, eps_pre=1e-6)
    assert (out == 0).all() and (n == 0).all()
    out, n = fn.flashnorm_block_residual(z, z, g_post=one, g_pre=one)
    assert torch.isnan(out).all() and torch.isnan(n).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_rows(fn, dtype):
    e = torch.empty(0, 64, dtype=dtype, device=DEV)
    one = torch.ones(64, device=DEV)
    out, n = fn.flashnorm_block_residual(e, e, g_post=one, g_pre=one, gate=e, rows_per_gate=4)
    assert out.shape == (0, 64) and n.shape == (0, 64)
    dx, dh, dgate, dpost, dpre = fn.flashnorm_block_residual_bwd(e, e, e, e, g_post=one, g_pre=one, gate=e, rows_per_gate=4)
    assert dx.shape == dh.shape == dgate.shape == (0, 64)
    assert (dpost == 0).all() and (dpre == 0).all()


@pytest.mark.parametrize("M,K,T", [(1, 4096, 0), (40, 576, 7), (1300, 264, 650)])
def test_repeats_graph_and_stream(fn, M, K, T):
    v = make(M, K, torch.bfloat16, True, T, True, seed=6)
    kw = kwargs(v, T, 1.0, 0.5)
    ins = [v[n].to(DEV) for n in ("x", "h", "dh_out", "dn")]

    def both(stream=None):
        return fn.flashnorm_block_residual(*ins[:2], stream=stream, **kw) + \
            fn.flashnorm_block_residual_bwd(*ins, stream=stream, **kw)

    same = lambda a, b: all(p is q is None or torch.equal(p, q) for p, q in zip(a, b))
    ref = both()
    assert same(both(), ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = both(side)
    side.synchronize()
    assert same(other, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        for t, n in zip(ins, ("x", "h", "dh_out", "dn")):
            t.copy_(make(M, K, torch.bfloat16, True, T, True, seed=7 + i)[n].to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert same(both(), held), i


def test_refusals_of_the_binding(fn):
    x = torch.ones(4, 64, device=DEV)
    one = torch.ones(64, device=DEV)
    call = fn.flashnorm_block_residual
    for bad in (lambda: call(x, x[:3]), lambda: call(x, x.bfloat16()), lambda: call(x, x.cpu()), lambda: call(x.cpu(), x.cpu()),
                lambda: call(x, x, g_post=one[:32]), lambda: call(x, x, g_post=one.bfloat16()),
                lambda: call(x, x, gate=x, rows_per_gate=2), lambda: call(x, x, gate=x, rows_per_gate=0),
                lambda: call(x, x, gate=x.bfloat16()), lambda: call(x, x, normed=torch.empty_like(x)),
                lambda: call(x, x, out=torch.empty(4, 72, device=DEV)), lambda: call(x.t(), x.t()),
                lambda: fn.flashnorm_block_residual_bwd(x, x, x[:2])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        call(x.half(), x.half())
    h = torch.ones(5, 64, device=DEV)
    for bad in (lambda: call(x, torch.ones_like(x), out=x), lambda: call(x, h[:4], out=h[1:]),
                lambda: call(x, torch.ones_like(x), eps_post=-1.0, g_post=one),
                lambda: call(torch.ones(2, 16388, device=DEV), torch.ones(2, 16388, device=DEV)),
                lambda: call(torch.ones(2, 66, device=DEV)[:, :62], torch.ones(2, 66, device=DEV)[:, :62]),
                lambda: fn.flashnorm_block_residual_bwd(x, x, None),
                lambda: fn.flashnorm_block_residual_bwd(x, x, x, None, g_pre=one),
                lambda: fn.flashnorm_block_residual_bwd(x, x, x, x)):
        with pytest.raises(fn.FlashNormError):
            bad()
