"""4-bit products: a call for every workgroup shape of both kernels, with every group size, kind and epilogue on it,
against 64-bit products (tolerances of test_w4.py); the kernels' register use and the LDS-DMA contract; two captured
graphs on one workspace; calls on two streams at once."""
import ctypes

import pytest
import torch

import __graft_entry__ as graft
from _codeobj import disassemble, kernel_resources
from test_lds_dma_m0 import m0_violations
from test_w4 import EPS, check, dense

DEV = "cuda:0"
SOURCES = [f"w4_{kernel}_{kind}.hip" for kernel in ("few", "many") for kind in ("rms", "glu", "row")]


class Plan(ctypes.Structure):
    _fields_ = [("many", ctypes.c_bool), ("shape", ctypes.c_int), ("splits", ctypes.c_int), ("kb_per_split", ctypes.c_int)]


def plan(M, K, N, glu, group, gs):
    """The kernel and workgroup shape that the built library takes for a call."""
    from paper_2407_09577_amd import flashnorm as fn
    graft.ensure_built()
    choose = getattr(fn.lib(), "_ZN2fn7w4_planEiiiibib")
    choose.argtypes, choose.restype = [ctypes.c_int] * 4 + [ctypes.c_bool, ctypes.c_int, ctypes.c_bool], Plan
    return choose(M, K, -(-K // 128), 2 * ((N // 2 + 15) // 16 * 16) if glu else (N + 15) // 16 * 16, glu, group, gs)


# (shape, plain M, K, N, GLU M, K, 2 F): K ends inside a block of 128, columns inside a block of 16, rows inside 16.
FEW = [  # read straight from memory, then staged through LDS (kW4StagedM rows and more)
    (0, (1, 144, 41), (3, 144, 42)), (0, (6, 528, 4226), (16, 544, 42)), (1, (5, 528, 13261), (1, 536, 8552)),
    (1, (7, 552, 13041), (6, 560, 8198)), (2, (1, 520, 16445), (2, 552, 16618)), (2, (6, 528, 17272), (9, 520, 16596)),
    (3, (1, 152, 8408), (4, 152, 8678)), (3, (15, 144, 8623), (6, 144, 9720)), (4, (2, 144, 16472), (1, 144, 16696)),
    (4, (6, 144, 17033), (13, 144, 17208)), (5, (17, 568, 12459), (17, 536, 12624)), (6, (17, 520, 16743), (18, 536, 17102)),
    (7, (1, 2072, 41), None), (7, (6, 2232, 41), None), (8, (1, 1056, 41), None), (8, (11, 1048, 41), None),
    (9, (1, 528, 8459), None), (9, (6, 520, 8225), None)]
MANY = [  # in one pass, then with K split
    (0, (492, 144, 21980), (770, 144, 14340)), (0, (100, 9544, 8258), (100, 10808, 8660)),
    (1, (338, 272, 16469), (338, 264, 16666)), (1, (102, 9408, 4114), (99, 9536, 4210)),
    (2, (391, 144, 20507), (399, 144, 19746)), (2, (67, 8232, 8218), (67, 8216, 9066)),
    (3, (82, 152, 21740), (449, 144, 4372)), (3, (67, 5352, 8305), (1177, 6176, 580)),
    (4, (52, 656, 16393), (51, 672, 16986)), (4, (50, 8664, 4126), (51, 10952, 2088)),
    (5, (53, 144, 21241), (49, 144, 20634)), (5, (37, 6232, 8657), (40, 6208, 8194)),
    (6, (86, 144, 17068), (83, 144, 16930)), (6, (17, 10480, 8346), (17, 10328, 4110)),
    (7, (1377, 2416, 524), (1399, 2344, 520)), (7, None, (683, 10520, 186)),
    (8, (71, 696, 21789), (67, 728, 21978)), (8, (82, 10352, 2895), (82, 10552, 2730)),
    (9, (97, 1248, 16842), (99, 912, 21834)), (9, (99, 8728, 4438), (98, 8296, 4158)),
    (10, None, None), (10, None, (17, 10672, 42))]
# Calls that go this way with a run-time g, or without one in groups of 32, as the few-row kernel is slower there.
MANY_G = [(7, True, (33, 10424, 290), False), (10, False, (1368, 2184, 133), False), (10, False, (1402, 3144, 66), True),
          (10, True, (17, 9640, 41), False)]
MANY_32 = [(7, True, (20, 10392, 2093), False), (10, False, (1374, 4120, 135), False), (10, False, (1391, 4136, 136), True),
           (10, True, (18, 11072, 40), False)]
CALLS = [(False, i % 2 == 1, s, c, glu) for i, (s, *cs) in enumerate(FEW) for glu, c in enumerate(cs) if c] + \
        [(True, i % 2 == 1, s, c, glu) for i, (s, *cs) in enumerate(MANY) for glu, c in enumerate(cs) if c]


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_shape_has_its_calls(group):
    assert {s for s, *_ in FEW} == set(range(10)) and {s for s, *_ in MANY} == set(range(11))
    for many, split, shape, call, glu in CALLS:
        for gs in (False, True):
            p = plan(*call, bool(glu), group, gs)
            if not many and (shape in (5, 6, 8) and gs or shape == 6 and group < 128):
                assert p.many or p.shape != shape  # no registers for these
                continue
            assert (p.many, p.shape) == (many, shape), (call, glu, gs)
            if many:
                assert (p.splits > 1) == split, call
    for shape, split, call, glu in MANY_G + (MANY_32 if group == 32 else []):
        p = plan(*call, glu, group, (shape, split, call, glu) in MANY_G)
        assert p.many and p.shape == shape and (p.splits > 1) == split, call


@pytest.mark.parametrize("source", SOURCES + ["w4_linear.hip", "w4_fold.hip", "residual.hip"])
def test_no_spills_in_loops(source, tmp_path):
    """No registers in scratch memory, but for one or two values that are stored before a kernel's loop and fetched
    behind it, and for fp32 gradients of rows of more than 8192 columns (four vectors a thread), which are known to."""
    res = kernel_resources(source, tmp_path)
    assert res
    long_rows = [n for n in res if "residual_bwd_kernelIfLi1024ELi4E" in n]
    assert [n for n, f in res.items() if f.get("sgpr_spill_count", 0) or f.get("vgpr_spill_count", 0) > 2
            and n not in long_rows] == []


@pytest.mark.parametrize("source", SOURCES)
def test_m0_only_feeds_lds_dma(source, tmp_path):
    ins = disassemble(source, tmp_path)
    assert len(ins) > 1000
    assert any(t.startswith("buffer_load") and t.endswith(" lds") for t in ins) == ("many" in source)
    assert m0_violations(ins) == []


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return flashnorm


def make(fn, M, K, N, glu, group, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    codes = torch.randint(0, 16, (K, N), generator=gen, dtype=torch.uint8, device=DEV)
    G = -(-K // group)
    scales = ((torch.rand(G, N, generator=gen, device=DEV) + 0.5) * K ** -0.5 / 4).to(torch.bfloat16)
    z = torch.randint(0, 16, (G, N), generator=gen, dtype=torch.uint8, device=DEV)
    a = torch.randn(M, K, generator=gen, device=DEV)
    a[::7] *= 20.0
    w4 = fn.pack_weights_w4(codes, scales, z, group=group, layout=fn.FN_LAYOUT_GLU if glu else fn.FN_LAYOUT_LINEAR)
    s = scales.double().repeat_interleave(group, 0)[:K]
    zz = z.double().repeat_interleave(group, 0)[:K]
    return a.to(torch.bfloat16), w4, (codes.double() - zz) * s, 8.0 * s.abs()


def ref_of(a, W, T, g=None, scale=None):
    x = a.double()
    s = (EPS + x.square().mean(1, keepdim=True)).rsqrt() if scale is None else scale.double()[:, None]
    if g is not None:
        x = x * g.double()
    mag = 2.0 ** -13 * (x.abs() @ T) * s.abs() + 1.5 * 2.0 ** -11 * (x.abs() @ W.abs()) * s.abs()
    return (x @ W) * s, mag


def padded(M, n):
    """An output inside a wider buffer, and a check that the rest stayed as it was."""
    buf = torch.full((M + 2, (n + 7) // 8 * 8 + 16), 3.0, dtype=torch.bfloat16, device=DEV)

    def kept():
        rest = buf.clone()
        rest[1:-1, 8:n + 8] = 3.0
        return bool((rest == 3.0).all())
    return buf[1:-1, 8:n + 8], kept


@pytest.mark.gpu
@pytest.mark.parametrize("many,split,shape,call,glu", CALLS + [(True, *c[1::-1], c[2], c[3]) for c in MANY_G + MANY_32])
def test_every_shape(fn, many, split, shape, call, glu):
    M, K, N = call
    for group in (32, 64, 128):
        a, w4, W, T = make(fn, M, K, N, glu, group, M + K + N + group)
        wide = torch.full((M, K + 16), float("nan"), dtype=torch.bfloat16, device=DEV)
        wide[:, 8:K + 8] = a
        x = wide[:, 8:K + 8]
        g = torch.rand(K, device=DEV) + 0.5
        for gg in (None, g):
            ref, mag = ref_of(a, W, T, gg)
            what = (call, group, gg is not None)
            if glu:
                F = N // 2
                out, kept = padded(M, F)
                fn.flashnorm_glu_w4(x, w4, EPS, g=gg, out=out)
                t, u, et, eu = ref[:, :F], ref[:, F:], mag[:, :F], mag[:, F:]
                ref = t * torch.sigmoid(t) * u
                tol = (2.0 ** -8 + 2.0 ** -20) * ref.abs() + 1.1 * et * (u.abs() + eu) + t.abs() * eu
            else:
                out, kept = padded(M, N)
                bias = torch.randn(N, device=DEV)
                fn.flashnorm_linear_w4(x, w4, EPS, g=gg, bias=bias, out=out)
                ref = ref + bias.double()
                tol = 2.0 ** -8 * ref.abs() + mag + 2.0 ** -23 * bias.abs()
            check(out, ref.cpu(), tol.cpu(), what)
            assert kept(), what
        if not glu:
            scale = torch.randn(M, device=DEV)
            out, kept = padded(M, N)
            fn.rowscale_linear_w4(x, w4, row_scale=scale, out=out)
            ref, mag = ref_of(a, W, T, scale=scale)
            check(out, ref.cpu(), (2.0 ** -8 * ref.abs() + mag).cpu(), (call, group, "row scale"))
            assert kept()


@pytest.mark.gpu
def test_two_graphs_on_one_workspace(fn):
    """Two captured calls that share a workspace, replayed in turn on one stream: each leaves the other nothing."""
    K, N = 2056, 5000
    a1, w1, *_ = make(fn, 300, K, N, False, 64, 1)
    a2, w2, *_ = make(fn, 280, K, N, False, 64, 2)
    size = fn.lib().flashnorm_w4_workspace_size
    need = max(size(M, K, N, 0, 64) for M in (300, 280))
    assert plan(300, K, N, False, 64, False).many and plan(280, K, N, False, 64, False).many
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    want1, want2 = fn.flashnorm_linear_w4(a1, w1, EPS), fn.flashnorm_linear_w4(a2, w2, EPS)
    out1, out2 = torch.empty_like(want1), torch.empty_like(want2)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph, a, w, out in ((graphs[0], a1, w1, out1), (graphs[1], a2, w2, out2)):
        with torch.cuda.graph(graph):
            fn.flashnorm_linear_w4(a, w, EPS, out=out, workspace=ws)
    for i in range(6):
        out1.zero_()
        out2.zero_()
        for j in ((0, 1), (1, 0), (0, 0, 1))[i % 3]:
            graphs[j].replay()
        torch.cuda.synchronize()
        assert torch.equal(out1, want1) and torch.equal(out2, want2), i


@pytest.mark.gpu
def test_two_streams_at_once(fn):
    """Calls in flight on two streams, with the workspaces that the binding allocates for each."""
    K, N = 2056, 1000
    a, w4, *_ = make(fn, 500, K, N, False, 128, 3)
    cases = [a, a[:200], a[:40], a[:16], a[:1]]
    want = [fn.flashnorm_linear_w4(x, w4, EPS) for x in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for i in range(20):
        with torch.cuda.stream(streams[i % 2]):
            got.append(fn.flashnorm_linear_w4(cases[i % 5], w4, EPS))
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 5]), i
