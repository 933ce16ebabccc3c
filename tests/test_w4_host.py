"""Host-side checks of the 4-bit weights and the block residual: sizes and refusals (no kernel launches)."""
import pytest

import __graft_entry__ as graft

A, W, Y, X, B = 0x100000, 0x10000000, 0x20000000, 0x30000000, 0x40000000


@pytest.fixture(scope="module")
def lib():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    return flashnorm.lib()


def test_size(lib):
    f = lib.fold_weights_w4_size
    # half a byte per weight of the padded shape, four bytes per group and packed column and four per column
    assert f(4096, 11008, 0, 128) == 4096 * 11008 // 2 + (32 + 1) * 11008 * 4
    assert f(4096, 11008, 0, 32) == 4096 * 11008 // 2 + (128 + 1) * 11008 * 4
    assert f(8, 3, 0, 128) == 128 * 16 // 2 + (1 + 1) * 16 * 4
    assert f(136, 2 * 9, 1, 64) == 256 * 32 // 2 + (4 + 1) * 32 * 4
    for bad in ((0, 16, 0, 32), (16, 0, 0, 32), (16, 7, 1, 32), (16, 16, 2, 32), (16, 16, 0, 48), (16, 16, 0, 0),
                (1 << 16, 1 << 16, 0, 128), ((1 << 21) + 8, 16, 0, 128)):
        assert f(*bad) == 0, bad


def _lin(lib, a=A, M=4, K=64, lda=64, adt=1, g=0, w=W, N=32, group=32, eps=1e-6, bias=0, y=Y, ldy=32, ydt=1, inv=0, ws=0,
         wb=0):
    return lib.flashnorm_linear_w4(a, M, K, lda, adt, g, w, N, group, eps, bias, y, ldy, ydt, inv, ws, wb, None)


def test_products_refuse(lib):
    assert _lin(lib, M=-1) == -2
    assert _lin(lib, K=0) == -2
    assert _lin(lib, K=60) == -2
    assert _lin(lib, N=0) == -2
    assert _lin(lib, lda=56) == -2
    assert _lin(lib, ldy=24) == -2
    assert _lin(lib, a=0) == -1
    assert _lin(lib, w=0) == -1
    assert _lin(lib, y=0) == -1
    assert _lin(lib, a=A + 8) == -4
    assert _lin(lib, w=W + 8) == -4
    assert _lin(lib, g=X + 4) == -4
    assert _lin(lib, bias=X + 4) == -4
    assert _lin(lib, inv=X + 2) == -4
    assert _lin(lib, lda=68) == -4
    assert _lin(lib, adt=7, ydt=7) == -3
    assert _lin(lib, adt=1, ydt=0) == -3
    assert _lin(lib, adt=0, ydt=0) == -5           # fp32 activations
    assert _lin(lib, group=48) == -6
    assert _lin(lib, eps=-1.0) == -6
    assert _lin(lib, eps=float("nan")) == -6
    assert _lin(lib, y=A + 64) == -8
    assert _lin(lib, y=W) == -8
    assert _lin(lib, g=Y) == -8
    assert _lin(lib, bias=Y) == -8
    assert _lin(lib, inv=Y) == -8
    assert _lin(lib, inv=A) == -8
    assert _lin(lib, lda=1 << 22) == -9
    big = dict(M=1 << 30, K=8, lda=8, N=1 << 20, ldy=1 << 20, y=1 << 60)
    assert _lin(lib, ws=1 << 61, wb=1 << 59, **big) == -9   # more workgroups than a launch takes
    wide = dict(M=1000, K=1024, lda=1024, N=8192, ldy=8192)   # such calls need a workspace
    assert _lin(lib, **wide) == -1
    need = lib.flashnorm_w4_workspace_size(1000, 1024, 8192, 0, 32)
    assert need > 1000 * 1024 * 2
    assert _lin(lib, ws=B, wb=need - 1, **wide) == -9
    assert _lin(lib, ws=B + 8, wb=need, **wide) == -4
    assert _lin(lib, ws=Y, wb=need, **wide) == -8 and _lin(lib, ws=A, wb=need, **wide) == -8
    f = lib.flashnorm_w4_workspace_size
    assert f(16, 4096, 4096, 0, 128) == 0 and f(0, 64, 32, 0, 32) == 0 and f(-1, 64, 32, 0, 32) == 0
    assert f(1000, 64, 31, 1, 32) == 0 and f(1000, 64, 32, 0, 16) == 0
    assert _lin(lib, M=0, a=0, y=0) == 0
    glu = lambda F=16, ldo=16, w=W: lib.flashnorm_glu_w4(A, 4, 64, 64, 1, None, w, F, 32, 1e-6, Y, ldo, 1, None, 0, None)
    assert glu(F=0) == -2 and glu(ldo=8) == -2 and glu(w=0) == -1
    row = lambda rs=0, y=Y: lib.rowscale_linear_w4(A, 4, 64, 64, 1, W, 32, 32, rs, y, 32, 1, None, 0, None)
    assert row(y=A) == -8 and row(rs=Y) == -8 and row(rs=X + 2) == -4


def test_folds_refuse(lib):
    f = lambda **k: lib.fold_weights_w4(k.get("W", A), k.get("sk", 32), k.get("sn", 1), k.get("dt", 1), k.get("g", 0),
                                        k.get("K", 64), k.get("N", 32), k.get("layout", 0), k.get("group", 32),
                                        k.get("zp", 0), k.get("out", Y), None)
    assert f(W=0) == -1 and f(out=0) == -1
    assert f(dt=4) == -3
    assert f(K=0) == -2 and f(N=0) == -2 and f(sk=-1) == -2 and f(N=31, layout=1) == -2
    assert f(layout=5) == -6 and f(group=16) == -6 and f(zp=2) == -6
    assert f(out=Y + 8) == -4 and f(W=A + 1) == -4
    assert f(sk=1 << 40) == -9 and f(K=1 << 22) == -9
    assert f(out=A) == -8 and f(g=Y) == -8
    p = lambda **k: lib.pack_weights_w4(k.get("q", A), k.get("ldc", 32), k.get("s", X), k.get("lds", 32), k.get("z", 0),
                                        k.get("ldz", 32), 64, 32, 0, k.get("group", 32), k.get("out", Y), None)
    assert p(q=0) == -1 and p(s=0) == -1 and p(out=0) == -1
    assert p(ldc=31) == -2 and p(lds=8) == -2 and p(z=B, ldz=8) == -2
    assert p(group=0) == -6
    assert p(out=Y + 4) == -4 and p(s=X + 2) == -4
    assert p(out=A) == -8 and p(s=Y) == -8 and p(z=Y) == -8
    u = lambda **k: lib.unpack_weights_w4(k.get("w", W), 64, 32, 0, k.get("group", 32), k.get("out", Y), k.get("ldo", 32), None)
    assert u(w=0) == -1 and u(out=0) == -1 and u(ldo=8) == -2 and u(group=7) == -6 and u(out=W) == -8 and u(out=Y + 2) == -4


def _res(lib, x=A, ldx=64, h=W, ldh=64, M=4, K=64, dt=1, gp=0, ep=1e-6, gate=0, ldg=64, T=1, rs=1.0, bs=1.0, gn=0, en=1e-6,
         out=Y, ldo=64, n=0, ldn=64, inv=0):
    return lib.flashnorm_block_residual(x, ldx, h, ldh, M, K, dt, gp, ep, gate, ldg, T, rs, bs, gn, en, out, ldo, n, ldn, inv,
                                        None)


def test_residual_refuses(lib):
    nan = float("nan")
    assert _res(lib, M=-1) == -2 and _res(lib, K=0) == -2 and _res(lib, K=60) == -2 and _res(lib, ldx=56) == -2
    assert _res(lib, K=16392, ldx=16392, ldh=16392, ldo=16392) == -9
    assert _res(lib, x=0) == -1 and _res(lib, h=0) == -1 and _res(lib, out=0) == -1
    assert _res(lib, n=X) == -1                                   # normed without g_pre
    assert _res(lib, dt=3) == -3
    assert _res(lib, x=A + 8) == -4 and _res(lib, gp=X + 4) == -4 and _res(lib, gate=B + 2) == -4 and _res(lib, ldx=68) == -4
    assert _res(lib, inv=X + 2) == -4
    assert _res(lib, gate=B, T=0) == -2
    assert _res(lib, ep=-1.0) == -6 and _res(lib, en=nan) == -6 and _res(lib, rs=nan) == -6 and _res(lib, bs=float("inf")) == -6
    assert _res(lib, out=A) == -8                                 # out may be h, not x
    assert _res(lib, out=W, ldo=72) == -8                         # h with another pitch
    assert _res(lib, out=W + 128) == -8                           # h shifted by a row
    assert _res(lib, out=Y, n=Y, gn=X) == -8 and _res(lib, gate=Y) == -8 and _res(lib, gp=Y) == -8 and _res(lib, inv=Y) == -8
    assert _res(lib, inv=A) == -8
    assert _res(lib, M=0, x=0, h=0, out=0) == 0


def _bwd(lib, x=A, h=W, do=X, dn=0, M=4, K=64, dt=1, gp=0, gate=0, T=1, gn=0, dx=Y, dh=Y + 0x10000, dg=0, dgp=0, dgn=0,
         ws=B, wb=1 << 20):
    return lib.flashnorm_block_residual_bwd(x, K, h, K, do, K, dn, K, M, K, dt, gp, 1e-6, gate, K, T, 1.0, 1.0, gn, 1e-6, dx, K,
                                            dh, K, dg, K, dgp, dgn, ws, wb, None)


def test_residual_bwd_refuses(lib):
    G, N, D = 0x50000000, 0x60000000, 0x70000000
    assert _bwd(lib, x=0) == -1 and _bwd(lib, h=0) == -1 and _bwd(lib, dx=0) == -1 and _bwd(lib, dh=0) == -1
    assert _bwd(lib, do=0) == -1                                  # no gradient at all
    assert _bwd(lib, gn=G) == -1                                  # g_pre without dn
    assert _bwd(lib, dn=N) == -1                                  # dn without g_pre
    assert _bwd(lib, dg=D) == -1 and _bwd(lib, dgp=D) == -1 and _bwd(lib, dgn=D) == -1   # gradients of nothing
    assert _bwd(lib, gp=G, dgp=D, ws=0) == -1
    assert _bwd(lib, gp=G, dgp=D, wb=15) == -9
    assert _bwd(lib, K=60) == -2 and _bwd(lib, gate=G, T=0) == -2
    assert _bwd(lib, dt=9) == -3 and _bwd(lib, ws=B + 4) == -4
    assert _bwd(lib, dx=A) == -8 and _bwd(lib, dh=W) == -8 and _bwd(lib, dh=Y) == -8 and _bwd(lib, gp=G, dgp=G) == -8
    assert _bwd(lib, gp=G, dgp=D, ws=Y) == -8
    assert _bwd(lib, M=0, x=0, h=0, do=0, dx=0, dh=0) == 0
    f = lib.flashnorm_block_residual_bwd_size
    assert f(4, 64, 0, 1) >= 2 * 64 * 4 and f(0, 64, 0, 1) > 0
    assert f(4, 60, 0, 1) == 0 and f(-1, 64, 0, 1) == 0 and f(4, 64, 0, 5) == 0 and f(4, 16392, 0, 1) == 0 and f(4, 64, -1, 1) == 0
