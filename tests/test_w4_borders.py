"""4-bit folds where rounding a product g w to fp32 would decide otherwise than the product itself: zero points and
codes next to a half, scales next to the border of two 12-bit values.  The definition (test_w4.quantise, 64 bits) has
to be met exactly, as everywhere else; random weights come to such a border once in a million groups or less."""
import numpy as np
import pytest
import torch

import __graft_entry__ as graft
from test_w4 import quantise

DEV = "cuda:0"


@pytest.fixture(scope="module")
def fn():
    graft.ensure_built()
    from paper_2407_09577_amd import flashnorm
    flashnorm.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return flashnorm


def bf16(x):
    return torch.as_tensor(x).to(torch.bfloat16).double().numpy()


def pair(rng, target, dtype):
    """w of the type and g of fp32 with |w| in [1, 2) and g w within 2 units in the last place of the target."""
    w = 1.0 + rng.random()
    w = float(bf16(np.float32(w))) if dtype == torch.bfloat16 else float(np.float32(w))
    g = np.float32(target / w)
    for _ in range(rng.integers(3)):
        g = np.nextafter(g, np.float32(rng.choice((-np.inf, np.inf))))
    return w, g


def borders(kind, K, group, dtype, zero_points, seed):
    """[K, 12] weights and g whose groups each come to one border, or one for each element ("code"); the columns are
    the same but for a power of two."""
    rng = np.random.default_rng(seed)
    w, g = np.zeros(K), np.ones(K, np.float32)
    for k0 in range(0, K, group):
        n = min(group, K - k0)
        # The scale that the definition rounds to, 12 bits, and one that rounds to it.
        d = rng.integers(2048, 4095) / 2048.0
        span = d + rng.uniform(-0.9, 0.9) / 4096.0
        if kind == "scale":  # next to the border between d and its neighbour
            span = d + 1.0 / 4096.0
        p, q = k0 + rng.choice(n, 2, replace=False)
        if zero_points:
            half = rng.integers(15) + 0.5
            # -lo / d next to a half; or anywhere, and the span then as it should be
            low = half * d if kind == "zero" else rng.uniform(0.2, 14.8) * d
            if kind == "scale":  # lo of few bits, so that hi - lo comes to the border
                low = float(bf16(np.float32(low)))
            w[p], g[p] = pair(rng, low, dtype)
            w[p] = -w[p]
            low = -w[p] * float(g[p])
            w[q], g[q] = pair(rng, 15.0 * span - low, dtype)
            zero = np.rint(low / d)
        else:
            w[p], g[p] = pair(rng, 7.0 * span, dtype)
            w[p] *= rng.choice((-1, 1))
            zero = 8
        if kind != "code":
            continue
        for k in set(range(k0, k0 + n)) - {p, q} if zero_points else set(range(k0, k0 + n)) - {p}:
            j = rng.integers(-zero, 15 - zero) if zero_points else rng.integers(-7, 7)
            t = (j + 0.5) * d
            w[k], g[k] = pair(rng, abs(t), dtype)
            w[k] *= np.sign(t)
    W = torch.from_numpy(w[:, None] * np.exp2(np.arange(-6, 6))).to(dtype)
    assert np.array_equal(W.double().numpy()[:, 6], w)
    return W, torch.from_numpy(g)


def undecided(W, g, group, zero_points):
    """How many elements of the first column the definition gives otherwise from products rounded to fp32."""
    rounded = (W[:, :1].float() * g[:, None]).double()
    return int((quantise(rounded, None, group, zero_points) != quantise(W[:, :1], g, group, zero_points)).sum())


CASES = [("zero", True), ("scale", False), ("scale", True), ("code", False), ("code", True)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind,zero_points", CASES)
def test_the_inputs_lie_at_borders(kind, zero_points, dtype):
    for K, group in ((1024, 32), (6400, 128)):
        W, g = borders(kind, K, group, dtype, zero_points, 1)
        assert undecided(W, g, group, zero_points) >= K // group // 8, (kind, K, group)


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("view", ["rows", "t", "third"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind,zero_points", CASES)
def test_fold_at_borders(fn, kind, zero_points, dtype, view, group):
    for K in (1000, 1024, 6400):  # whole columns in a workgroup, and not
        W, g = borders(kind, K, group, dtype, zero_points, K + group)
        if view == "t":
            Wd = W.t().contiguous().to(DEV).t()
        elif view == "third":
            Wd = torch.zeros(K, 3 * W.shape[1], dtype=dtype, device=DEV)[:, 1::3]
            Wd.copy_(W)
        else:
            Wd = W.to(DEV)
        w4 = fn.fold_weights_w4(Wd, g.to(DEV), group=group, zero_points=zero_points)
        got = fn.unpack_weights_w4(w4).cpu().double().numpy()
        ref = quantise(W, g, group, zero_points)
        assert np.array_equal(got, ref), (K, np.abs(got - ref).max(), int((got != ref).sum()))


# Two values of a group (the others are zeros) whose zero point is 7, while the smaller product rounded to fp32 makes it
# 8: -lo is just below 7.5 scales, and the scale is not the span that it is rounded from.
PINNED = [((-1.5546875, 0.24600541591644287), (1.9296875, 0.19824708998203278)),
          ((-(7.5 + 14 * 2.0 ** -21), 1 - 15 * 2.0 ** -24), (7.5 + 15 * 2.0 ** -13, 1.0))]


@pytest.mark.gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("view", ["rows", "t"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_zero_points_below_a_half(fn, dtype, view, group):
    for i, ((w0, g0), (w1, g1)) in enumerate(PINNED):
        if dtype == torch.bfloat16 and i == 1:
            continue  # w0 has more bits
        K = 2 * group
        w, g = torch.zeros(K, dtype=torch.float64), torch.ones(K)
        w[1], g[1], w[30], g[30] = w0, g0, w1, g1
        w[group + 17], g[group + 17], w[group + 2], g[group + 2] = w0, g0, w1, g1
        W = (w[:, None] * torch.exp2(torch.arange(-6, 6))).to(dtype)
        ref = quantise(W, g, group, True)
        s = ref[30] / 8
        assert np.array_equal(ref[1], -7 * s) and np.array_equal(ref[group + 2], 8 * s)
        Wd = W.to(DEV) if view == "rows" else W.t().contiguous().to(DEV).t()
        got = fn.unpack_weights_w4(fn.fold_weights_w4(Wd, g.to(DEV), group=group, zero_points=True)).cpu().double().numpy()
        assert np.array_equal(got, ref), i
