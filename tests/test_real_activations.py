"""The operators on real activations with packed weights (linear_bits, gated_bits) and the norms around them (norm_residual),
forwards and backwards, against their definitions in 64 bits on the CPU.

Tolerances are bounds, derived per element from what the operators promise: sums in float32 (relative error of a sum
of n products at most (n + 8) 2^-24 of the sum of their magnitudes), activations to a few float32 units, one rounding to
the result's type (relative 2^-8 bfloat16, 2^-11 float16, 2^-24 float32, absolute half of the smallest subnormal), and backwards
one more rounding of the gradient before the scale."""
import math

import numpy as np
import pytest
import torch

import paper_1602_02830_amd as bnn
from paper_1602_02830_amd import binding

DEV = "cuda:0"
gpu = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}
F32 = 2.0 ** -24
ACTS = {"none": bnn.ACT_NONE, "relu": bnn.ACT_RELU, "silu": bnn.ACT_SILU, "gelu": bnn.ACT_GELU, "gelu_tanh": bnn.ACT_GELU_TANH,
        "sigmoid": bnn.ACT_SIGMOID}
NORMS = {"none": bnn.NORM_NONE, "rms": bnn.NORM_RMS, "layer": bnn.NORM_LAYER}


def phi(z, act):
    """An activation and its derivative, float64."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.clamp(z, min=0), (z > 0).double()
    if act == "gelu":
        c = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * c, c + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return (s, s * (1 - s)) if act == "sigmoid" else (z * s, s + z * s * (1 - s))


class Product:
    """Operands of a product on the CPU and on the GPU.  Rows lie `gap` elements apart beyond their length and start `shift`
    elements into a buffer whose other elements are NaN; weights have junk in pad bits and pad words."""

    def __init__(self, M, N, K, T, scale=True, bias=True, gap=0, shift=0, seed=0, x_std=1.0):
        g = torch.Generator().manual_seed(1000 * seed + M + 7 * N + 31 * K)
        self.T, self.gap, self.shift = T, gap, shift
        self.x = (torch.randn(M, K, generator=g) * x_std).to(T)
        self.w = torch.randint(0, 2, (N, K), generator=g).mul_(2).sub_(1).double()
        self.scale = (torch.rand(N, generator=g) + 0.5) / math.sqrt(max(K, 1)) if scale else None
        self.bias = 0.3 * torch.randn(N, generator=g) if bias else None
        self.xd = self.place(self.x)
        words = (K + 31) // 32
        bits = np.zeros((N, words * 32), np.uint8)
        bits[:, :K] = self.w.numpy() > 0
        bits[:, K:] = 1
        packed = np.packbits(bits, axis=1, bitorder="little").view(np.uint32).reshape(N, words)
        buf = np.full((N, words + (3 if gap else 0)), 0x5A5A5A5A, np.uint32)
        buf[:, :words] = packed
        self.wd = torch.from_numpy(buf.view(np.int32)).to(DEV)[:, :words]
        self.scaled = self.scale.to(DEV) if scale else None
        self.biased = self.bias.to(DEV) if bias else None

    def place(self, t, gap=None):
        rows, cols = t.shape
        gap = self.gap if gap is None else gap
        buf = torch.full((rows * (cols + gap) + self.shift + 8,), float("nan"), dtype=self.T, device=DEV)
        v = buf[self.shift:self.shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
        v.copy_(t)
        return v

    def z(self, w=None):
        """s, z and bounds of the errors of both."""
        x, w = self.x.double(), self.w
        K = x.shape[1]
        s = x @ w.t()
        es = (K + 8) * F32 * (x.abs().sum(1, keepdim=True).expand_as(s))
        a = self.scale.double() if self.scale is not None else torch.ones(w.shape[0], dtype=torch.float64)
        b = self.bias.double() if self.bias is not None else torch.zeros(w.shape[0], dtype=torch.float64)
        z = s * a + b
        return s, es, a, z, es * a + 4 * F32 * (z.abs() + b.abs() + (s * a).abs())


def act_error(z, ez, act):
    """Bound of the error of phi(z) and of its derivative, computed from a z with error ez: slopes of all activations and
    of their derivatives are below 1.2; evaluation errors below 32 float32 units of max(1, |z|) (of |z| + 1 sums of a few terms)."""
    if act == "none":
        return ez, torch.zeros_like(ez)
    ev = 32 * F32 * (1 + z.abs())
    jump = (z.abs() <= ez).double() if act == "relu" else 0.0
    return 1.2 * ez + (0 if act == "relu" else ev), 1.2 * ez + (0 if act == "relu" else ev) + jump


def close(got, want, tol, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), (got - want)[bad].abs().max().item(), tol.expand_as(want)[bad].min().item())


def rounded(want, err, T):
    return err + ROUND[T] * (want.abs() + err) + TINY[T]


def linear_want(p, act, residual=None):
    s, es, a, z, ez = p.z()
    f, _ = phi(z, act)
    ef, _ = act_error(z, ez, act)
    if residual is not None:
        f = f + residual.double()
        ef = ef + F32 * f.abs()
    return f, rounded(f, ef, p.T)


def gated_want(p, act):
    s, es, a, z, ez = p.z()
    F = z.shape[1] // 2
    f, _ = phi(z[:, :F], act)
    ef, _ = act_error(z[:, :F], ez[:, :F], act)
    zu, eu = z[:, F:], ez[:, F:]
    h = f * zu
    eh = f.abs() * eu + zu.abs() * ef + ef * eu + F32 * h.abs()
    return h, rounded(h, eh, p.T)


LINEAR_SIZES = [(1, 1, 1), (1, 33, 31), (2, 32, 32), (3, 100, 33), (17, 130, 257), (31, 64, 100), (32, 5, 1000), (33, 33, 33),
                (64, 128, 64), (100, 257, 127), (129, 129, 129), (200, 320, 513), (300, 96, 4096), (5, 300, 4100)]


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M,N,K", LINEAR_SIZES)
def test_linear(M, N, K, T):
    T = TYPES[T]
    p = Product(M, N, K, T)
    r = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(T)
    got = bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_NONE, r.to(DEV))
    close(got, *linear_want(p, "none", r), "linear")
    got = bnn.linear_bits(p.xd, p.wd, p.scaled, None, bnn.ACT_SILU)
    p.bias = None
    close(got, *linear_want(p, "silu"), "linear silu")


# Sizes whose tiles fill the chip in each of the tiled forms (64, 128 and 256 rows), with partial tiles, steps and words.
@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M,N,K", [(1000, 4090, 100), (2040, 4090, 70), (4090, 4090, 65), (4000, 4096, 640), (300, 20000, 7)])
def test_linear_large_tiles(M, N, K, T):
    T = TYPES[T]
    p = Product(M, N, K, T, seed=2, gap=1 if K == 65 else 0)
    r = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(T)
    close(bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_NONE, r.to(DEV)), *linear_want(p, "none", r), "large")


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M,F,K", [(1000, 2045, 100), (2040, 2045, 70), (4090, 2045, 65)])
def test_gated_large_tiles(M, F, K, T):
    p = Product(M, 2 * F, K, TYPES[T], seed=2)
    close(bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU), *gated_want(p, "silu"), "large")


@gpu
@pytest.mark.parametrize("M", [5, 40, 130])
def test_rows_far_apart(M):
    """Rows more than 2^23 elements apart: a tile's offsets need 64 bits."""
    K, N, ld = 70, 20480, 2 ** 23 + 9
    p = Product(M, N, K, torch.bfloat16)
    far = torch.empty((M - 1) * ld + K, dtype=torch.bfloat16, device=DEV).as_strided((M, K), (ld, 1))
    far.copy_(p.x)
    close(bnn.linear_bits(far, p.wd, p.scaled, p.biased), *linear_want(p, "none"), "far")
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).mul_(0.1).bfloat16()
    got = bnn.linear_bits_backward(dy.to(DEV), far, p.wd, p.scaled, p.biased, bnn.ACT_SILU)
    check_backward(p, "silu", False, dy, got)


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [7, 70])
def test_linear_activations(M, act, T):
    p = Product(M, 70, 190, TYPES[T], seed=3)
    p.scale *= 4                                   # z reaches the tails
    p.scaled *= 4
    close(bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, ACTS[act]), *linear_want(p, act), act)


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("gap,shift", [(0, 1), (1, 0), (5, 3), (8, 8), (3, 0)])
@pytest.mark.parametrize("M,N,K", [(3, 45, 77), (140, 200, 136), (70, 65, 128)])
def test_linear_strides_and_alignment(M, N, K, gap, shift, T):
    T = TYPES[T]
    p = Product(M, N, K, T, gap=gap, shift=shift)
    r = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(T)
    rd, out = p.place(r), p.place(torch.zeros(M, N), gap=2 * gap)
    around = out._base if out._base is not None else out
    before = torch.isnan(around).sum()
    got = bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU, rd, out=out)
    assert got is out
    close(out, *linear_want(p, "gelu", r), "strided")
    assert torch.isnan(around).sum() == before                      # nothing written between or behind the rows
    got = bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU, rd, out=rd)      # in the residual's place
    assert torch.equal(got, out)


# Rows of 16-bit elements that begin inside a 32-bit word, all of them or every other one, and end anywhere; what lies around them is NaN.
@gpu
@pytest.mark.parametrize("T", ["bf16", "f16"])
@pytest.mark.parametrize("gap,shift", [(0, 0), (0, 1), (1, 0), (1, 1), (2, 1), (7, 3)])
@pytest.mark.parametrize("M,K", [(3, 2047), (5, 1025), (16, 1536), (11, 2050), (20, 257), (40, 512), (70, 775), (33, 1279)])
def test_rows_that_begin_inside_a_word(M, K, gap, shift, T):
    T = TYPES[T]
    p = Product(M, 150, K, T, seed=13, gap=gap, shift=shift)
    close(bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU), *linear_want(p, "gelu"), "linear")
    close(bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU), *gated_want(p, "silu"), "gated")


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "sigmoid", "none"])
@pytest.mark.parametrize("M,F,K", [(1, 1, 1), (1, 40, 100), (2, 33, 4100), (32, 64, 64), (33, 31, 65), (130, 65, 200), (257, 200, 96)])
def test_gated(M, F, K, act, T):
    p = Product(M, 2 * F, K, TYPES[T], seed=5)
    close(bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased, ACTS[act]), *gated_want(p, act), act)


@gpu
@pytest.mark.parametrize("gap,shift", [(1, 0), (0, 1), (8, 8)])
@pytest.mark.parametrize("M", [4, 150])
def test_gated_strides(M, gap, shift):
    p = Product(M, 2 * 77, 131, torch.float16, bias=False, gap=gap, shift=shift)
    out = p.place(torch.zeros(M, 77), gap=gap)
    bnn.gated_bits(p.xd, p.wd, p.scaled, None, bnn.ACT_SILU, out=out)
    close(out, *gated_want(p, "silu"), "strided gated")


def backward_want(p, act, gated, dy):
    """Gradients and bounds.  ds is rounded to the type before the products; sums of rounding errors are bounded twice: every
    element by the sum of their bounds, the whole by three times what independent errors would give."""
    s, es, a, z, ez = p.z()
    T, x, w, u = p.T, p.x.double(), p.w, ROUND[p.T]
    d = dy.double()
    M, K = x.shape
    if gated:
        F = z.shape[1] // 2
        f, df = phi(z[:, :F], act)
        ef, edf = act_error(z[:, :F], ez[:, :F], act)
        zu, eu = z[:, F:], ez[:, F:]
        dz = torch.cat([d * zu * df, d * f], 1)
        edz = torch.cat([d.abs() * (zu.abs() * edf + df.abs() * eu + eu * edf), d.abs() * ef], 1) + 4 * F32 * dz.abs()
    else:
        _, df = phi(z, act)
        _, edf = act_error(z, ez, act)
        dz = d * df
        edz = d.abs() * edf + 2 * F32 * dz.abs()
    ds = dz * a
    first = 0.0 if not gated and act == "none" and p.scale is None else u
    eds = edz * a + first * (ds.abs() + edz * a) + TINY[T]
    n = ds.shape[1]
    dx, dw = ds @ w, ds.t() @ x
    rel_n, rel_m = (n + 8) * F32, (M + 8) * F32
    edx = eds.sum(1, keepdim=True).expand_as(dx) + rel_n * ds.abs().sum(1, keepdim=True)
    edw = eds.t() @ x.abs() + rel_m * (ds.abs().t() @ x.abs())
    es_all = dz.abs() * es + edz * (s.abs() + es)
    want = {"dx": (dx, rounded(dx, edx, T)), "dw": (dw, rounded(dw, edw, T)),
            "dscale": ((dz * s).sum(0), es_all.sum(0) + (M + K + 8) * F32 * (d.abs() if not gated and act == "none" else dz.abs()).t()
                       .mul((x.abs().sum(1)).unsqueeze(0)).sum(1)),
            "dbias": (dz.sum(0), edz.sum(0) + rel_m * dz.abs().sum(0))}
    spread = {"dx": ((u * ds) ** 2 / 3).sum(1, keepdim=True).expand_as(dx) + (u * dx) ** 2 / 3,
              "dw": (((u * ds) ** 2).t() @ (x * x)) / 3 + (u * dw) ** 2 / 3}
    return want, spread


def check_backward(p, act, gated, dy, got, parts=("dx", "dw", "dscale", "dbias")):
    want, spread = backward_want(p, act, gated, dy)
    for k in parts:
        close(got[k], *want[k], k)
    if p.T != torch.float32 and act != "relu":
        for k in ("dx", "dw"):
            if k in parts and want[k][0].numel() >= 256:
                err = (got[k].cpu().double() - want[k][0]).square().mean().sqrt()
                assert err <= 3 * spread[k].mean().sqrt() + 1e-6 * want[k][0].square().mean().sqrt(), (k, err)


BACK_SIZES = [(1, 1, 1), (1, 64, 33), (2, 33, 100), (33, 31, 31), (64, 64, 64), (100, 129, 130), (129, 200, 257), (300, 65, 128),
              (513, 140, 40)]


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ["none", "gelu", "relu"])
@pytest.mark.parametrize("M,N,K", BACK_SIZES)
def test_linear_backward(M, N, K, act, T):
    T = TYPES[T]
    p = Product(M, N, K, T, seed=7)
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    check_backward(p, act, False, dy, bnn.linear_bits_backward(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act]))


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid", "relu", "none"])
@pytest.mark.parametrize("M,F,K", [(1, 1, 1), (1, 33, 64), (40, 32, 100), (130, 65, 129), (257, 100, 70)])
def test_gated_backward(M, F, K, act, T):
    T = TYPES[T]
    p = Product(M, 2 * F, K, T, seed=9)
    dh = torch.randn(M, F, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    check_backward(p, act, True, dh, bnn.gated_bits_backward(dh.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act]))


# Tiles of 64, 128 and 256 rows with their column sums, and the weights' gradient in tiles of 64 (whole and in parts of the rows),
# 128 and 256.
@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("M,N,K", [(1000, 4090, 100), (2040, 4090, 70), (4090, 4090, 65), (70, 4090, 3100), (40, 2100, 2000), (4000, 100, 90),
                                   (1500, 3, 5), (70, 5, 300), (70, 300, 5)])
def test_linear_backward_large_tiles(M, N, K, act, T):
    T = TYPES[T]
    p = Product(M, N, K, T, seed=7)
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    check_backward(p, act, False, dy, bnn.linear_bits_backward(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act]))


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M,F,K", [(200, 1500, 1101), (90, 2900, 1300)])
def test_products_in_tiles_of_128_channels_without_lds(M, F, K, T):
    T = TYPES[T]
    p = Product(M, 2 * F, K, T, seed=15)
    close(bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU), *linear_want(p, "gelu"), "linear")
    close(bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU), *gated_want(p, "silu"), "gated")
    for gated in (False, True):
        dy = torch.randn(M, F if gated else 2 * F, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
        f = bnn.gated_bits_backward if gated else bnn.linear_bits_backward
        check_backward(p, "silu", gated, dy, f(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU))


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("M,N,K", [(6000, 300, 521), (9001, 131, 255), (700, 300, 200), (2100, 1030, 260)])
def test_linear_backward_parts_of_the_rows(M, N, K, act, T):
    """The weights' gradient joined from parts of the rows, in tiles of 64 and of 128."""
    T = TYPES[T]
    p = Product(M, N, K, T, seed=7)
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    check_backward(p, act, False, dy, bnn.linear_bits_backward(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act]))


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M,F,K", [(1000, 2045, 100), (2040, 2045, 70), (4090, 2045, 65), (70, 2045, 3100), (3000, 50, 90)])
def test_gated_backward_large_tiles(M, F, K, T):
    T = TYPES[T]
    p = Product(M, 2 * F, K, T, seed=9)
    dh = torch.randn(M, F, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    check_backward(p, "silu", True, dh, bnn.gated_bits_backward(dh.to(DEV), p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU))


@gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("gap,shift", [(1, 0), (0, 1), (8, 8)])
def test_backward_strides_and_no_vectors(gap, shift, act, gated):
    T = torch.bfloat16
    M, N, K = 150, 154, 131
    p = Product(M, N, K, T, scale=False, bias=False, gap=gap, shift=shift, x_std=0.1)
    cols = N // 2 if gated else N
    dy = torch.randn(M, cols, generator=torch.Generator().manual_seed(2)).to(T)
    call = bnn.gated_bits_backward if gated else bnn.linear_bits_backward
    got = call(p.place(dy), p.xd, p.wd, None, None, ACTS[act])
    assert got["dscale"] is None and got["dbias"] is None
    check_backward(p, act, gated, dy, got, ("dx", "dw"))
    some = call(p.place(dy), p.xd, p.wd, None, None, ACTS[act], need_dx=False)
    assert some["dx"] is None and torch.equal(some["dw"], got["dw"])
    some = call(p.place(dy), p.xd, p.wd, None, None, ACTS[act], need_dw=False)
    assert some["dw"] is None and torch.equal(some["dx"], got["dx"])


@gpu
def test_weights_gradient_is_what_flipping_a_bit_does():
    """Without an activation the loss sum(dy * y) is linear in the weights: flipping w[n][k] changes it by -2 w dw[n][k]."""
    p = Product(37, 45, 70, torch.float32, seed=4)
    dy = torch.randn(37, 45, generator=torch.Generator().manual_seed(2))
    dw = bnn.linear_bits_backward(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased)["dw"].cpu().double()
    base = (bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased).cpu().double() * dy).sum()
    for n, k in ((0, 0), (44, 69), (17, 33), (31, 31), (32, 32)):
        w = p.wd.clone()
        bit = np.int64(w[n, k // 32].item()) & 0xFFFFFFFF ^ (1 << (k % 32))
        w[n, k // 32] = int(np.uint32(bit).view(np.int32))
        diff = (bnn.linear_bits(p.xd, w, p.scaled, p.biased).cpu().double() * dy).sum() - base
        # two float32 losses of 1665 terms of magnitude about 1: each term within 80 * 2^-24 of its size
        assert abs(diff + 2 * p.w[n, k] * dw[n, k]) < 1665 * 80 * F32 * 2


@gpu
@pytest.mark.parametrize("gated", [False, True])
def test_gradients_against_differences(gated):
    """Central differences of the float32 forward pass in random directions of x, scale and bias.  With a step of 2^-7 the
    third-order term is below 1e-4 of the directional derivative's scale, and the losses' rounding (80 float32 units of each of
    3000 terms, independent) below 1e-4 of it too; 2e-3 of the scale is asked."""
    M, N, K = 50, 120, 60
    p = Product(M, N, K, torch.float32, seed=6)
    cols = N // 2 if gated else N
    dy = torch.randn(M, cols, generator=torch.Generator().manual_seed(2))
    fwd = bnn.gated_bits if gated else bnn.linear_bits
    back = bnn.gated_bits_backward if gated else bnn.linear_bits_backward
    got = back(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU)
    args = {"dx": p.xd, "dscale": p.scaled, "dbias": p.biased}
    for name, t in args.items():
        v = torch.randn(t.shape, generator=torch.Generator().manual_seed(8)).to(DEV) * t.abs().mean()
        step = 2.0 ** -7
        losses = []
        for sign in (1, -1):
            moved = {k: (a + sign * step * v if k == name else a) for k, a in args.items()}
            y = fwd(moved["dx"], p.wd, moved["dscale"], moved["dbias"], bnn.ACT_GELU)
            losses.append((y.cpu().double() * dy).sum())
        diff = (losses[0] - losses[1]) / (2 * step)
        g = got[name].cpu().double()
        assert abs(diff - (g * v.cpu().double()).sum()) <= 2e-3 * (g.norm() * v.cpu().double().norm()), name


@gpu
@pytest.mark.parametrize("T", TYPES)
def test_empty_products(T):
    T = TYPES[T]
    x = torch.randn(3, 0, device=DEV).to(T)
    w = torch.empty(6, 0, dtype=torch.int32, device=DEV)
    scale, bias = torch.ones(6, device=DEV), torch.arange(6.0, device=DEV)
    assert torch.equal(bnn.linear_bits(x, w, scale, bias, bnn.ACT_RELU), bias.to(T).expand(3, 6))
    h = bnn.gated_bits(x, w, scale, bias, bnn.ACT_NONE)
    assert torch.equal(h, (bias[:3] * bias[3:]).to(T).expand(3, 3))
    got = bnn.linear_bits_backward(torch.ones(3, 6, device=DEV).to(T), x, w, scale, bias)
    assert got["dx"].shape == (3, 0) and got["dw"].shape == (6, 0)
    assert torch.equal(got["dscale"], torch.zeros(6, device=DEV)) and torch.equal(got["dbias"], torch.full((6,), 3.0, device=DEV))
    got = bnn.gated_bits_backward(torch.ones(3, 3, device=DEV).to(T), x, w, scale, bias, bnn.ACT_NONE)
    assert torch.equal(got["dbias"], 3 * torch.cat([bias[3:], bias[:3]])) and not got["dscale"].any()
    # no rows: gradients of the parameters are zero
    w = torch.ones(6, 2, dtype=torch.int32, device=DEV)
    e = torch.empty(0, 40, dtype=T, device=DEV)
    assert bnn.linear_bits(e, w).shape == (0, 6) and bnn.gated_bits(e, w).shape == (0, 3)
    for got in (bnn.linear_bits_backward(torch.empty(0, 6, dtype=T, device=DEV), e, w, scale, bias),
                bnn.linear_bits_backward(torch.empty(0, 6, dtype=T, device=DEV), e, w, scale, bias, bnn.ACT_SILU),
                bnn.gated_bits_backward(torch.empty(0, 3, dtype=T, device=DEV), e, w, scale, bias)):
        assert got["dx"].shape == (0, 40) and not got["dw"].any() and not got["dscale"].any() and not got["dbias"].any()
    # no channels: the gradient of x is zero
    none = torch.empty(0, 2, dtype=torch.int32, device=DEV)
    x = torch.randn(3, 40, device=DEV).to(T)
    assert bnn.linear_bits(x, none).shape == (3, 0)
    assert not bnn.linear_bits_backward(torch.empty(3, 0, dtype=T, device=DEV), x, none)["dx"].any()


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M", [2, 80])
def test_infinities_and_nans_stay_in_their_rows(M, T):
    T = TYPES[T]
    p = Product(M, 70, 133, T)
    p.xd[0, 3] = float("inf")
    p.xd[1, 5] = float("nan")
    got = bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased).float().cpu()
    assert torch.equal(got[0], torch.where(p.w[:, 3] > 0, float("inf"), float("-inf")).float())
    assert torch.isnan(got[1]).all()
    want, tol = linear_want(p, "none")
    if M > 2:
        close(got[2:], want[2:], tol[2:], "other rows")


@gpu
def test_float32_rows_as_exact_as_float32_products():
    """Values over the whole range of magnitudes in one row: the three terms of each keep all of its 24 bits."""
    p = Product(40, 40, 96, torch.float32, scale=False, bias=False)
    p.x *= torch.exp2(torch.randint(-20, 20, p.x.shape, generator=torch.Generator().manual_seed(1)).float())
    p.xd.copy_(p.x)
    close(bnn.linear_bits(p.xd, p.wd), *linear_want(p, "none"), "range")
    one = torch.zeros(40, 96)
    one[:, 7] = torch.randn(40, generator=torch.Generator().manual_seed(1)) * 1e30
    one[0, 7] = torch.finfo(torch.float32).max
    got = bnn.linear_bits(one.to(DEV), p.wd).cpu()
    assert torch.equal(got, one[:, 7:8] * p.w[:, 7].float())


@gpu
def test_products_repeat_and_take_other_streams():
    p = Product(300, 200, 500, torch.bfloat16)
    dh = torch.randn(300, 100, device=DEV).bfloat16()
    first = bnn.gated_bits_backward(dh, p.xd, p.wd, p.scaled, p.biased)
    again = bnn.gated_bits_backward(dh, p.xd, p.wd, p.scaled, p.biased)
    for k in first:
        assert torch.equal(first[k], again[k]), k
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = bnn.gated_bits_backward(dh, p.xd, p.wd, p.scaled, p.biased)
        h = bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased)
    side.synchronize()
    for k in first:
        assert torch.equal(first[k], other[k]), k
    assert torch.equal(h, bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased))


@gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "silu", "sigmoid"])
@pytest.mark.parametrize("dy_std", [1e-3, 1e-4, 1e-5, 1e-6])
@pytest.mark.parametrize("M,N,K", [(12, 1024, 200), (70, 2048, 130), (300, 4096, 96)])
def test_float16_backward_keeps_small_gradients(M, N, K, dy_std, act, gated):
    """dy far below 1 and a channel scale of 1/64: dz * scale lies among float16's subnormals, or below them.  The error is that of
    roundings relative to 2^-11 alone (three times what independent ones give in the mean square), and of a result's own end."""
    p = Product(M, N, K, torch.float16, seed=17)
    p.scale = (torch.rand(N, generator=torch.Generator().manual_seed(5)) + 0.5) / 64
    p.scaled = p.scale.to(DEV)
    cols = N // 2 if gated else N
    dy = torch.randn(M, cols, generator=torch.Generator().manual_seed(2)).mul_(dy_std).half()
    call = bnn.gated_bits_backward if gated else bnn.linear_bits_backward
    got = call(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act])
    want, spread = backward_want(p, act, gated, dy)
    for k in ("dx", "dw"):
        err = (got[k].cpu().double() - want[k][0]).square().mean().sqrt()
        bound = 3 * (spread[k].mean() + TINY[p.T] ** 2 / 3).sqrt() + 1e-6 * want[k][0].square().mean().sqrt()
        assert err <= bound, (k, err.item(), bound.item(), want[k][0].square().mean().sqrt().item())


@gpu
@pytest.mark.parametrize("act", ["silu", "sigmoid"])
@pytest.mark.parametrize("M,F,K,loud", [(64, 256, 1024, 1000), (64, 256, 1024, 10000), (1500, 33, 300, 1000), (40, 300, 4, 1000)])
def test_float16_backward_beside_loud_rows(M, F, K, loud, act):
    """Some rows of x and others of dh have elements far above the rest: the other rows keep their digits, by the row's mean square."""
    p = Product(M, 2 * F, K, torch.float16, seed=21)
    p.scale = (torch.rand(2 * F, generator=torch.Generator().manual_seed(5)) + 0.5) / 64
    p.scaled = p.scale.to(DEV)
    dh = torch.randn(M, F, generator=torch.Generator().manual_seed(2)).mul_(1e-3)
    p.x[:2, :40] = (p.x[:2, :40].float() * loud).clamp(-6e4, 6e4).half()
    p.xd.copy_(p.x)
    dh[2:4, :10] *= loud
    dh = dh.half()
    got = bnn.gated_bits_backward(dh.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act])["dx"].cpu().double()
    want, spread = backward_want(p, act, True, dh)
    want, spread = want["dx"][0][4:], spread["dx"][4:]
    err = (got[4:] - want).square().mean(1).sqrt()
    bound = 3 * (spread.mean(1) + TINY[p.T] ** 2 / 3).sqrt() + 1e-6 * want.square().mean(1).sqrt()
    assert (err <= bound).all(), (err / bound).max().item()


@gpu
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_float16_backward_of_large_gradients(act, gated):
    """Gradients up to float16's largest, an infinite one and a NaN in rows of their own: the others are as they are without them."""
    M, N, K = 70, 64, 2000
    p = Product(M, N, K, torch.float16, seed=19)
    cols = N // 2 if gated else N
    dy = torch.randn(M, cols, generator=torch.Generator().manual_seed(2)).mul_(1e4).clamp_(-65504, 65504).half()
    dy[3, 5] = 65504.0
    call = bnn.gated_bits_backward if gated else bnn.linear_bits_backward
    got = call(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act])
    check_backward(p, act, gated, dy, got, ("dx",))
    dy[1, 2], dy[2, 7] = float("inf"), float("nan")
    spoilt = call(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act])
    assert not torch.isfinite(spoilt["dx"][1:3]).any()
    want = backward_want(p, act, gated, dy)[0]["dx"]
    rows = [0] + list(range(3, M))
    close(spoilt["dx"][rows], want[0][rows], want[1][rows], "other rows")


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("act", ["gelu", "sigmoid"])
def test_tails_of_activations_keep_their_digits(act, T):
    """One product of one element a row, so that z is exact.  Relative to the result: a few units of the functions, and what a unit in
    the exponent's argument (z^2 / 2, or z) makes of them."""
    T = TYPES[T]
    z = torch.cat([torch.linspace(-12, 12, 193), torch.linspace(-3, 20, 47)]).to(T)
    w = torch.ones(1, 1, dtype=torch.int32, device=DEV)
    x = z.unsqueeze(1).to(DEV)
    z64 = z.double().unsqueeze(1)
    f, df = phi(z64, act)
    df = df if act == "gelu" else torch.exp(-z64) / (1 + torch.exp(-z64)) ** 2
    # Of the derivative of gelu's two terms, which have opposite signs below zero, the sum of the magnitudes.
    size = 0.5 * torch.special.erfc(-z64 / math.sqrt(2)) + z64.abs() * torch.exp(-0.5 * z64 ** 2) / math.sqrt(2 * math.pi) if act == "gelu" else df
    units = (16 + 2 * (z64 ** 2 if act == "gelu" else z64.abs())) * F32
    close(bnn.linear_bits(x, w, act=ACTS[act]), f, rounded(f, units * f.abs(), T), act)
    got = bnn.linear_bits_backward(torch.ones_like(x), x, w, act=ACTS[act])["dx"]
    err = units * size
    close(got, df, rounded(df, err + ROUND[T] * (df.abs() + err), T), "slope")


@gpu
@pytest.mark.parametrize("M,N,K", [(40, 70, 90), (9001, 131, 255), (70, 5, 300)])
def test_infinities_in_the_weights_gradient(M, N, K):
    """float32: what an infinity is multiplied with has terms that are zero."""
    p = Product(M, N, K, torch.float32, seed=23, scale=False, bias=False)
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2))
    dy[2:6] = torch.tensor([1.0, -0.5, 0.75, 3.0]).unsqueeze(1)             # of few bits
    dy[2, 1] = 0.0
    inf = float("inf")
    p.x[2, 7], p.x[3, 8], p.x[30, 9] = inf, -inf, inf                          # by the few bits, by any number
    p.x[4, 10], p.x[5, 10] = inf, inf                                          # of one sign each: infinite
    p.x[6], dy[6, 3], dy[31, 4] = 2.0, -inf, inf
    p.x[6, 11], p.x[31, 12] = inf, 0.0
    p.xd.copy_(p.x)
    dw = bnn.linear_bits_backward(dy.to(DEV), p.xd, p.wd)["dw"].cpu().double()
    want = dy.double().t() @ p.x.double()
    assert torch.equal(torch.isnan(dw), torch.isnan(want)) and torch.isnan(want).any()
    there = ~torch.isnan(want)
    assert torch.equal(torch.isinf(dw[there]), torch.isinf(want[there])) and torch.isinf(want).sum() > 2 * N
    inside = torch.isinf(want)
    assert torch.equal(dw[inside], want[inside])
    fin = torch.isfinite(want)
    clean = torch.where(torch.isfinite(p.x), p.x, 0.0).double(), torch.where(torch.isfinite(dy), dy, 0.0).double()
    tol = (M + 8) * F32 * (clean[1].abs().t() @ clean[0].abs())
    close(dw[fin], want[fin], rounded(want[fin], tol[fin], torch.float32), "finite")


# More than four rows and 8192 columns: two blocks of 16 channels a workgroup (gated: four), of one wavefront or several, with rows that begin
# anywhere.
@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("gap,shift", [(0, 0), (1, 1)])
@pytest.mark.parametrize("M,N,K", [(5, 8192, 70), (16, 8209, 1500), (5, 8209, 4100), (16, 8192, 2051)])
def test_few_rows_of_many_channels(M, N, K, gap, shift, T):
    T = TYPES[T]
    p = Product(M, N, K, T, seed=31, gap=gap, shift=shift)
    r = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(T)
    close(bnn.linear_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU, r.to(DEV)), *linear_want(p, "gelu", r), "linear")
    p = Product(M, 2 * N, K, T, seed=31, gap=gap, shift=shift)
    close(bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU), *gated_want(p, "silu"), "gated")


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,N,K", [(5, 8192, 70), (16, 8209, 1100)])
def test_backward_of_few_rows_of_many_channels(M, N, K, gated, T):
    T = TYPES[T]
    p = Product(M, N * (1 + gated), K, T, seed=31, gap=1)
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    call = bnn.gated_bits_backward if gated else bnn.linear_bits_backward
    check_backward(p, "silu", gated, dy, call(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, bnn.ACT_SILU))


# The weights' gradient in tiles of 128 in parts of the rows, of 256 (16 bits) and 128 (float32) in parts, and of 256 and 128 in one part of more
# steps than buffers; in the second the products are tiles of 256 and 128 rows with weights past 512 and 1024 elements.
@gpu
@pytest.mark.parametrize("M,N,K,T", [(3001, 1100, 700, "bf16"), (3001, 1100, 700, "f16"), (3001, 1100, 700, "f32"), (4090, 4090, 1100, "bf16"),
                                     (4090, 4090, 1100, "f32"), (520, 4000, 4080, "f16"), (520, 4000, 4080, "f32")])
@pytest.mark.parametrize("form", ["linear none", "linear silu", "gated silu"])
def test_backward_in_large_tiles_of_many_steps(M, N, K, T, form):
    T = TYPES[T]
    kind, act = form.split()
    p = Product(M, N, K, T, seed=33)
    if kind == "gated":
        dh = torch.randn(M, N // 2, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
        close(bnn.gated_bits(p.xd, p.wd, p.scaled, p.biased, ACTS[act]), *gated_want(p, act), "forwards")
        return check_backward(p, act, True, dh, bnn.gated_bits_backward(dh.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act]))
    dy = torch.randn(M, N, generator=torch.Generator().manual_seed(2)).mul_(0.1).to(T)
    check_backward(p, act, False, dy, bnn.linear_bits_backward(dy.to(DEV), p.xd, p.wd, p.scaled, p.biased, ACTS[act]))


# ---- norms -------------------------------------------------------------------------------------------------------

class Norm:
    def __init__(self, M, D, R, T, post, pre, x=True, gate=True, gap=0, seed=0):
        g = torch.Generator().manual_seed(1000 * seed + M + 7 * D)
        self.T, self.M, self.D, self.R, self.post, self.pre = T, M, D, R, post, pre
        self.y = (torch.randn(M, D, generator=g) * 2 + 0.5).to(T)
        self.x = torch.randn(M, D, generator=g).to(T) if x else None
        self.gate = (1 + 0.3 * torch.randn(-(-M // R), D, generator=g)).to(T) if gate else None
        self.vec = {}
        for side, kind in (("post", post), ("pre", pre)):
            self.vec[side + "_gamma"] = 1 + 0.2 * torch.randn(D, generator=g) if kind != "none" else None
            self.vec[side + "_beta"] = 0.2 * torch.randn(D, generator=g) if kind == "layer" else None
        self.dr, self.dn = (torch.randn(M, D, generator=g).mul_(0.1).to(T) for _ in range(2))
        self.gap = gap

    def dev(self, t):
        if t is None:
            return None
        buf = torch.full((t.shape[0], t.shape[1] + self.gap), float("nan"), dtype=t.dtype, device=DEV)
        buf[:, :t.shape[1]] = t.to(DEV)
        return buf[:, :t.shape[1]]

    def call(self, **kw):
        v = {k: (t.to(DEV) if t is not None else None) for k, t in self.vec.items()}
        return bnn.norm_residual(self.dev(self.y), self.dev(self.x), self.dev(self.gate), 0.5, NORMS[self.post], v["post_gamma"],
                                 v["post_beta"], NORMS[self.pre], v["pre_gamma"], v["pre_beta"], 1e-5, self.R, **kw)

    def back(self, r, dr=True):
        v = {k: (t.to(DEV) if t is not None else None) for k, t in self.vec.items()}
        return bnn.norm_residual_backward(self.dev(self.dr) if dr else None, self.dev(self.dn) if self.pre != "none" else None,
                                          self.dev(self.y), self.dev(r), self.dev(self.gate), 0.5, NORMS[self.post], v["post_gamma"],
                                          v["post_beta"], NORMS[self.pre], v["pre_gamma"], v["pre_beta"], 1e-5, self.R,
                                          need_dx=self.x is not None)

    def leaves(self, r=None):
        """float64 leaves for torch's differentiation of the definition."""
        get = lambda t: None if t is None else t.double().requires_grad_(True)
        lv = {"y": get(self.y), "x": get(self.x), "gate": get(self.gate)}
        lv.update({k: get(t) for k, t in self.vec.items()})
        return lv


def norm64(v, kind, gamma, beta):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    h = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5) * gamma
    return h if beta is None else h + beta


def stream64(n, lv):
    t = norm64(lv["y"], n.post, lv["post_gamma"], lv["post_beta"])
    r = 0.5 * t
    if lv["gate"] is not None:
        r = r * lv["gate"].repeat_interleave(n.R, 0)[:n.M]
    return r if lv["x"] is None else lv["x"] + r


def norm_tol(want, T, D, scale):
    """One rounding, and float32 sums over D and a few operations on values up to `scale` (the largest magnitude a row
    passes through, amplified by 1 / sqrt(var), which is 1 here)."""
    return ROUND[T] * want.abs() + TINY[T] + (64 + math.sqrt(D)) * F32 * scale


NORM_SIZES = [(1, 1, 1), (1, 4096, 1), (3, 7, 2), (5, 100, 5), (4, 512, 1), (7, 513, 3), (40, 1024, 40), (33, 1025, 10), (9, 2050, 4),
              (6, 4100, 2), (3, 8200, 3), (2, 16384, 1), (3000, 65, 700), (2100, 24, 1)]


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "none"), ("none", "none")])
@pytest.mark.parametrize("M,D,R", NORM_SIZES)
def test_norm(M, D, R, post, pre, T):
    if D == 1 and "layer" in (post, pre):
        pytest.skip("a layer norm of one element is its beta: covered by test_layer_norm_of_one_element")
    n = Norm(M, D, R, TYPES[T], post, pre)
    r, nn = n.call()
    lv = n.leaves()
    with torch.no_grad():
        want = stream64(n, lv)
        scale = max(1.0, n.y.double().abs().max().item(), want.abs().max().item()) * 2
        close(r, want, norm_tol(want, n.T, D, scale), "r")
        if pre == "none":
            assert nn is None
        else:
            wn = norm64(want, pre, lv["pre_gamma"], lv["pre_beta"])
            amp = (1 / torch.sqrt(want.var(1, unbiased=False) + 1e-5)).max().item() if pre == "layer" else \
                  (1 / torch.sqrt((want * want).mean(1) + 1e-5)).max().item()
            close(nn, wn, norm_tol(wn, n.T, D, scale * max(1.0, amp) * 4), "n")


@gpu
def test_layer_norm_of_one_element():
    n = Norm(5, 1, 1, torch.float32, "layer", "layer")
    r, nn = n.call()
    assert torch.allclose(nn.cpu(), n.vec["pre_beta"].expand(5, 1), atol=0, rtol=0)


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("x,gate,gap", [(True, False, 0), (False, True, 1), (False, False, 8), (True, True, 3)])
def test_norm_operands_and_strides(x, gate, gap, T):
    n = Norm(37, 203, 10, TYPES[T], "layer", "rms", x=x, gate=gate, gap=gap)
    r, nn = n.call()
    lv = n.leaves()
    with torch.no_grad():
        want = stream64(n, lv)
        close(r, want, norm_tol(want, n.T, 203, 20.0), "r")
        wn = norm64(want, "rms", lv["pre_gamma"], None)
        close(nn, wn, norm_tol(wn, n.T, 203, 40.0), "n")
    if x:                                           # the stream's own place
        xd = n.dev(n.x)
        v = {k: (t.to(DEV) if t is not None else None) for k, t in n.vec.items()}
        r2, nn2 = bnn.norm_residual(n.dev(n.y), xd, n.dev(n.gate), 0.5, NORMS["layer"], v["post_gamma"], v["post_beta"], NORMS["rms"],
                                    v["pre_gamma"], None, 1e-5, n.R, out=xd)
        assert r2 is xd and torch.equal(r2, r) and torch.equal(nn2, nn)


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("rms", "none"), ("layer", "rms"), ("none", "none")])
@pytest.mark.parametrize("M,D,R", [s for s in NORM_SIZES if s[1] > 1] + [(1200, 80, 2), (1100, 600, 1100), (50, 12000, 25)])
def test_norm_backward(M, D, R, post, pre, T):
    n = Norm(M, D, R, TYPES[T], post, pre, seed=2)
    lv = n.leaves()
    r64 = stream64(n, lv)
    r = r64.detach().to(n.T)
    # Differentiated at the rounded stream, which is what the backward pass is given.
    rr = r64 + (r.double() - r64).detach()
    loss = (rr * n.dr.double()).sum()
    if pre != "none":
        loss = loss + (norm64(rr, pre, lv["pre_gamma"], lv["pre_beta"]) * n.dn.double()).sum()
    loss.backward()
    got = n.back(r)
    # Magnitudes that float32 errors are relative to: gradients of up to 8 through factors gamma / sqrt(var) of up to `amp`.
    ry = n.y.double()
    amp_y = (1 / torch.sqrt(((ry - ry.mean(1, keepdim=True)) if post == "layer" else ry).square().mean(1) + 1e-5)).max().item()
    rv = r.double()
    amp_r = (1 / torch.sqrt(((rv - rv.mean(1, keepdim=True)) if pre == "layer" else rv).square().mean(1) + 1e-5)).max().item()
    d_scale = 4 * (1 + (amp_r if pre != "none" else 0))
    y_scale = 4 * d_scale * (amp_y if post != "none" else 1)
    hat = 4 * max(1.0, math.log(M * D + 1))
    for name, key, scale in (("dx", "x", d_scale), ("dy", "y", y_scale)):
        want = lv[key].grad
        close(got[name], want, norm_tol(want, n.T, D, scale), name)
    want = lv["gate"].grad
    close(got["dgate"], want, norm_tol(want, n.T, D, d_scale * hat * min(R, M) ** 0.5) + (min(R, M) + 8) ** 0.5 * 4 * F32 * d_scale * hat, "dgate")
    for k in ("post_gamma", "post_beta", "pre_gamma", "pre_beta"):
        if n.vec[k] is None:
            assert got["d" + k] is None
        else:
            # a sum over M rows of float32 terms, in strips: errors of the terms add up like independent ones, times 8
            want = lv[k].grad
            scale = d_scale * hat
            close(got["d" + k], want, torch.full_like(want, 8 * (64 + math.sqrt(D)) * F32 * scale * math.sqrt(M)), "d" + k)
    if pre == "rms" and post == "rms":
        again = n.back(r)
        for k, v in got.items():
            assert v is None or torch.equal(v, again[k]), k


@gpu
def test_norm_backward_without_the_streams_gradient():
    n = Norm(30, 300, 7, torch.float32, "rms", "rms")
    r, _ = n.call()
    n.dr.zero_()
    with_zero, without = n.back(r.cpu()), n.back(r.cpu(), dr=False)
    for k, v in with_zero.items():
        assert v is None or torch.equal(v, without[k]), k


@gpu
def test_norm_rows_past_2_31_elements():
    """Offsets of more than 32 bits: a matrix of 4.3 GB whose last rows are looked at."""
    M, D = 2 ** 19 + 5, 4104
    y = torch.zeros(M, D, dtype=torch.bfloat16, device=DEV)
    y[-3:] = torch.randn(3, D, device=DEV).bfloat16()
    r, n = bnn.norm_residual(y, pre=bnn.NORM_RMS, rows_per_gate=M)
    assert torch.equal(r[-3:], y[-3:])
    want = norm64(y[-3:].cpu().double(), "rms", 1.0, None)
    close(n[-3:], want, norm_tol(want, torch.bfloat16, D, 20.0), "last rows")
    assert not n[:-3].any()


@gpu
def test_product_rows_past_2_31_elements():
    M, N, K = 2 ** 19 + 5, 40, 4104
    p = Product(3, N, K, torch.bfloat16)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    x[-3:] = p.xd
    y = bnn.linear_bits(x, p.wd, p.scaled, p.biased)
    close(y[-3:], *linear_want(p, "none"), "last rows")
    assert torch.equal(y[:-3], p.biased.bfloat16().expand(M - 3, N))


def strips(M, D, R):
    """Rows of a strip of the backward pass, and whether a gate is several of them (as the launcher has it)."""
    target = 4096 if D <= 512 else 2048 if D <= 1024 else 1024 if D <= 2048 else 512 if D <= 4096 else 256
    rows = -(-M // target)
    R = min(R, M)
    return (rows // R * R, False) if R <= rows else (-(-R // -(-R // rows)), True)


def walkers(D):
    """Workgroups of the forward pass, which walk over the rows."""
    threads = 64 if D <= 1024 else 64 * -(-D // 1024) if D <= 8192 else 1024
    return 256 * (1024 // threads)


@gpu
@pytest.mark.parametrize("gate_rows", ["1", "2", "above a strip", "700", "all"])
@pytest.mark.parametrize("M,D,T", [(9001, 7, "f32"), (9001, 65, "bf16"), (5000, 600, "f32"), (2501, 1500, "f16"), (2600, 2049, "f32"),
                                   (2600, 2049, "bf16"), (1700, 5000, "f16"), (700, 9000, "bf16"), (700, 9000, "f32")])
def test_norms_of_more_rows_than_workgroups(M, D, T, gate_rows):
    """A workgroup has several rows: the next one's loads, the gate's row that changes on the way, the sums over rows.  What belongs to
    a row is what the row gets by itself, bit for bit; the sums are compared with the definition."""
    T = TYPES[T]
    R = {"above a strip": strips(M, D, 1)[0] + 1, "all": M}.get(gate_rows) or int(gate_rows)
    rows, several = strips(M, D, R)
    assert M > walkers(D) and rows > 1 and several == (R > strips(M, D, 1)[0])
    post, pre = ("layer", "rms") if R % 2 else ("rms", "layer")
    n = Norm(M, D, R, T, post, pre, seed=6)
    dev = lambda t: None if t is None else t.to(DEV)
    v = {k: dev(t) for k, t in n.vec.items()}
    y, x, gate, dr, dn = dev(n.y), dev(n.x), dev(n.gate), dev(n.dr), dev(n.dn)
    per_row = gate.repeat_interleave(R, 0)[:M]
    post_args = (NORMS[post], v["post_gamma"], v["post_beta"])
    pre_args = (NORMS[pre], v["pre_gamma"], v["pre_beta"], 1e-5)
    r, nn = bnn.norm_residual(y, x, gate, 0.5, *post_args, *pre_args, R)
    got = bnn.norm_residual_backward(dr, dn, y, r, gate, 0.5, *post_args, *pre_args, R)
    for a in range(0, M, 200):                                         # as few rows as there are workgroups and strips for
        b = min(a + 200, M)
        assert strips(200, D, 1)[0] == 1 and walkers(D) >= 200
        own = bnn.norm_residual(y[a:b], x[a:b], per_row[a:b], 0.5, *post_args, *pre_args, 1)
        assert torch.equal(own[0], r[a:b]) and torch.equal(own[1], nn[a:b]), a
        back = bnn.norm_residual_backward(dr[a:b], dn[a:b], y[a:b], r[a:b], per_row[a:b], 0.5, *post_args, *pre_args, 1)
        assert torch.equal(back["dx"], got["dx"][a:b]) and torch.equal(back["dy"], got["dy"][a:b]), a
    # The definition in 64 bits, differentiated at the rounded stream.
    lv = {k: None if t is None else t.double().requires_grad_() for k, t in {"y": y, "x": x, "gate": gate, **v}.items()}
    r64 = stream64(n, lv)
    rr = r64 + (r.double() - r64).detach()
    hat_r = norm64(rr, pre, 1.0, None)
    ((rr * dr.double()).sum() + (norm64(rr, pre, lv["pre_gamma"], lv["pre_beta"]) * dn.double()).sum()).backward()
    # A term of a sum over rows is a gradient times a normalised element; float32 errors of either are units of the largest it was
    # made of (of the gradient: dr, and dn gamma / sqrt(var) of the row), and their sums' errors no more than all of them.
    unit = (64 + math.sqrt(D)) * F32
    with torch.no_grad():
        inv = 1 / torch.sqrt(((rr - rr.mean(1, keepdim=True)) if pre == "layer" else rr).square().mean(1, keepdim=True) + 1e-5)
        d, g = lv["x"].grad, 0.5 * per_row.double()
        d_size = d.abs() + dr.double().abs() + 3 * inv * (dn.double() * lv["pre_gamma"]).abs().amax(1, keepdim=True)
        hat_y = norm64(lv["y"], post, 1.0, None)
        t = norm64(lv["y"], post, lv["post_gamma"], lv["post_beta"])
        hat_size, y_size = hat_r.abs() + hat_r.abs().amax(1, keepdim=True), hat_y.abs() + hat_y.abs().amax(1, keepdim=True)
        by_gate = lambda s: torch.stack([s[a:a + R].sum(0) for a in range(0, M, R)])
        sums = {"dpre_gamma": (lv["pre_gamma"], (dn.double().abs() * hat_size).sum(0)), "dpre_beta": (lv["pre_beta"], dn.double().abs().sum(0)),
                "dpost_gamma": (lv["post_gamma"], (g.abs() * d_size * y_size).sum(0)), "dpost_beta": (lv["post_beta"], (g.abs() * d_size).sum(0))}
        for k, (leaf, size) in sums.items():
            assert (leaf is None) == (got[k] is None), k
            if leaf is not None:
                close(got[k], leaf.grad.cpu(), (unit * size).cpu(), k)
        want, err = lv["gate"].grad.cpu(), (unit * by_gate(0.5 * d_size * (t.abs() + t.abs().amax(1, keepdim=True)))).cpu()
        close(got["dgate"], want, rounded(want, err, T), "dgate")


@gpu
@pytest.mark.parametrize("T", TYPES)
def test_backward_calls_through_ctypes_and_natively(T, monkeypatch):
    T = TYPES[T]
    p = Product(90, 2 * 77, 131, T, gap=3, shift=1)
    n = Norm(50, 203, 10, T, "layer", "rms", gap=3)
    r = torch.randn(50, 203, generator=torch.Generator().manual_seed(5)).to(T)
    dy = p.place(torch.randn(90, 154, generator=torch.Generator().manual_seed(2)).to(T))
    assert binding.load_library() and binding._calls is not None

    def all_of_them():
        return [bnn.linear_bits_backward(dy, p.xd, p.wd, p.scaled, p.biased, bnn.ACT_GELU),
                bnn.linear_bits_backward(dy, p.xd, p.wd, p.scaled, need_dw=False),
                bnn.gated_bits_backward(dy[:, :77], p.xd, p.wd, p.scaled, None, bnn.ACT_SILU, need_dx=False), n.back(r)]

    natively = all_of_them()
    monkeypatch.setattr(binding, "_calls", None)
    for a, b in zip(natively, all_of_them()):
        assert a.keys() == b.keys()
        for k in a:
            assert (a[k] is None) == (b[k] is None) and (a[k] is None or torch.equal(a[k], b[k])), k


# ---- the block -------------------------------------------------------------------------------------------------------

def block64(x, n, w_in, w_out, s_in, s_out, gate, post_g, next_g, act):
    """BinaryFeedForward in float64 on the CPU, weights +-1 as given (leaves for differentiation)."""
    z = (n @ w_in.t()) * s_in
    F = z.shape[1] // 2
    y = ((phi(z[:, :F], act)[0] * z[:, F:]) @ w_out.t()) * s_out
    r = x + 0.7 * gate * norm64(y, "rms", post_g, None)
    return r, norm64(r, "rms", next_g, None)


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M", [1, 9, 200])
def test_block_forwards_and_backwards(M, T):
    T = TYPES[T]
    D, F = 96, 160
    g = torch.Generator().manual_seed(M)
    w_in, w_out = torch.randn(2 * F, D, generator=g) * 0.1, torch.randn(D, F, generator=g) * 0.1
    gammas = [1 + 0.1 * torch.randn(D, generator=g) for _ in range(3)]
    gate = (1 + 0.1 * torch.randn(1, D, generator=g)).to(T)
    x, dr, dn = (torch.randn(M, D, generator=g).to(T) for _ in range(3))
    block = bnn.BinaryFeedForward(w_in.to(DEV), w_out.to(DEV), bnn.ACT_SILU, *(v.to(DEV) for v in gammas), gate.to(DEV), 0.7)
    n = block.first_norm(x.to(DEV))
    r, after = block.forward(x.to(DEV), n, keep=True)
    dx, dn_in = block.backward(dr.to(DEV), dn.to(DEV))
    d = lambda t: t.double().requires_grad_(True)
    sign = lambda w: torch.where(w >= 0, 1.0, -1.0).double().requires_grad_(True)
    leaves = {"x": d(x), "n": d(n.cpu()), "w_in": sign(w_in), "w_out": sign(w_out), "scale_in": d(block.scale_in.cpu()),
              "scale_out": d(block.scale_out.cpu()), "gate": d(gate), "post_gamma": d(gammas[1]), "next_gamma": d(gammas[2])}
    want_n = norm64(leaves["x"].detach(), "rms", gammas[0].double(), None)
    close(n, want_n, norm_tol(want_n, T, D, 16.0), "first norm")
    wr, wa = block64(*leaves.values(), "silu")
    ((wr * dr.double()).sum() + (wa * dn.double()).sum()).backward()
    # h, y and r, and backwards dr's sum, dy, dh and ds, are rounded to the type on the way: eight roundings of values of the size of
    # their tensor, each of which reaches a result through factors of order one (norms divide by their size).
    def near(got, want, what):
        err = (got.detach().cpu().double() - want).norm() / want.norm()
        assert err <= 8 * ROUND[T] + 1e-5, (what, err)
    near(r, wr.detach(), "r")
    near(after, wa.detach(), "n'")
    near(dx, leaves["x"].grad, "dx")
    near(dn_in, leaves["n"].grad, "dn")
    for k in ("w_in", "w_out", "scale_in", "scale_out", "gate", "post_gamma", "next_gamma"):
        near(block.grads[k], leaves[k].grad, k)
    with pytest.raises(RuntimeError):
        block.forward(x.to(DEV), n)
        block.backward(dr.to(DEV), dn.to(DEV))


@gpu
def test_block_learns():
    """Straight-through training of the real weights lowers the loss: everything runs together as a program would use it."""
    g = torch.Generator().manual_seed(0)
    D, F, M = 64, 128, 256
    w_in, w_out = (0.1 * torch.randn(2 * F, D, generator=g)).to(DEV), (0.1 * torch.randn(D, F, generator=g)).to(DEV)
    block = bnn.BinaryFeedForward(w_in, w_out)
    x = torch.randn(M, D, generator=g).to(DEV)
    target = torch.tanh(x @ torch.randn(D, D, generator=g).to(DEV) / 8)
    n = block.first_norm(x)
    losses = []
    for _ in range(60):
        r, after = block.forward(x, n, keep=True)
        diff = r - x - target
        losses.append(diff.square().mean().item())
        block.backward(2 * diff / diff.numel(), torch.zeros_like(after))
        for w, k in ((w_in, "w_in"), (w_out, "w_out")):
            w -= 0.02 * block.grads[k] / (block.grads[k].abs().mean() + 1e-12) * w.abs().mean()
        block.set_weights(w_in, w_out)
    assert min(losses[-10:]) < 0.8 * losses[0], losses[::10]


def small_block(T=torch.bfloat16, gate=True, D=64, F=96):
    g = torch.Generator().manual_seed(3)
    w_in, w_out = (torch.randn(*s, generator=g).mul_(0.1).to(DEV) for s in ((2 * F, D), (D, F)))
    gate = (1 + 0.1 * torch.randn(1, D, generator=g)).to(T).to(DEV) if gate else None
    block = bnn.BinaryFeedForward(w_in, w_out, pre_gamma=torch.rand(D, generator=g).add_(0.5).to(DEV), gate=gate)
    x = torch.randn(20, D, generator=g).to(T).to(DEV)
    return block, x, (w_in, w_out)


@gpu
def test_block_with_new_weights_has_nothing_to_differentiate():
    block, x, (w_in, w_out) = small_block()
    r, after = block.forward(x, block.first_norm(x), keep=True)
    block.set_weights(-w_in, w_out)
    with pytest.raises(RuntimeError, match="forward"):
        block.backward(torch.ones_like(r), torch.zeros_like(after))


@gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("which", ["n", "r", "a view of r"])
def test_block_refuses_what_was_written_over(which, native, monkeypatch):
    """The stream and the normalised input are the caller's: written over in between, they would give wrong gradients."""
    block, x, _ = small_block()
    if not native:
        monkeypatch.setattr(binding, "_calls", None)
    n = block.first_norm(x)
    r, after = block.forward(x, n, keep=True)
    dr, dn = torch.ones_like(r), torch.zeros_like(after)
    block.backward(dr, dn)                                             # as they were: no complaint
    if which == "n":
        bnn.linear_bits(n, torch.ones(n.shape[1], 2, dtype=torch.int32, device=DEV), out=n.clone())       # read only
        block.backward(dr, dn)
        bnn.gated_bits(x, torch.ones(2 * n.shape[1], 2, dtype=torch.int32, device=DEV), out=n)
    else:
        out = r if which == "r" else r[3:7]
        bnn.norm_residual(dr[:out.shape[0]], out, out=out)             # the documented place of the next sum
    with pytest.raises(RuntimeError, match="written over"):
        block.backward(dr, dn)


@gpu
def test_block_in_inference_mode():
    block, x, _ = small_block()
    want = block.forward(x, block.first_norm(x))
    with torch.inference_mode():
        y = x.clone()
        got = block.forward(y, block.first_norm(y), keep=True)
        assert bnn.norm_residual(y, y, out=y)[0] is y
        block.backward(torch.ones_like(y), torch.zeros_like(y))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert bnn.norm_residual(x, x, out=y)[0] is y                      # an inference tensor outside of that mode


@gpu
@pytest.mark.parametrize("T", TYPES)
@pytest.mark.parametrize("M", [1, 50])
def test_block_gradient_through_the_first_norm(M, T):
    T = TYPES[T]
    D, F = 96, 160
    g = torch.Generator().manual_seed(M)
    w_in, w_out = torch.randn(2 * F, D, generator=g) * 0.1, torch.randn(D, F, generator=g) * 0.1
    gammas = [1 + 0.1 * torch.randn(D, generator=g) for _ in range(3)]
    gate = (1 + 0.1 * torch.randn(1, D, generator=g)).to(T)
    x, dr, dn = (torch.randn(M, D, generator=g).to(T) for _ in range(3))
    block = bnn.BinaryFeedForward(w_in.to(DEV), w_out.to(DEV), bnn.ACT_SILU, *(v.to(DEV) for v in gammas), gate.to(DEV), 0.7)
    xd = x.to(DEV)
    block.forward(xd, block.first_norm(xd), keep=True)
    dx, dn_in = block.backward(dr.to(DEV), dn.to(DEV))
    total = block.first_norm_backward(xd, dn_in, dx)
    alone = block.first_norm_backward(xd, dn_in)
    d = lambda t: t.double().requires_grad_(True)
    sign = lambda w: torch.where(w >= 0, 1.0, -1.0).double()
    lx, lg = d(x), d(gammas[0])
    n = norm64(lx, "rms", lg, None)
    wr, wa = block64(lx, n, sign(w_in), sign(w_out), block.scale_in.cpu().double(), block.scale_out.cpu().double(), gate.double(),
                     gammas[1].double(), gammas[2].double(), "silu")
    ((wr * dr.double()).sum() + (wa * dn.double()).sum()).backward()
    # As the block's other gradients, with two more roundings on the way: of n forwards and of its gradient backwards.
    for got, want, what in ((total, lx.grad, "dx"), (block.grads["pre_gamma"], lg.grad, "pre_gamma"), (total - alone, dx.cpu().double(), "sum")):
        err = (got.detach().cpu().double() - want).norm() / want.norm()
        assert err <= 10 * ROUND[T] + 1e-5, (what, err)


@gpu
@pytest.mark.parametrize("gate", [True, False])
def test_block_without_rows(gate):
    block, x, _ = small_block(gate=gate)
    e = x[:0]
    r, after = block.forward(e, block.first_norm(e), keep=True)
    assert r.shape == after.shape == e.shape
    dx, dn = block.backward(torch.empty_like(r), torch.empty_like(after))
    assert dx.shape == dn.shape == e.shape
    for k, v in block.grads.items():
        assert (v is None) == (k in ("post_gamma", "next_gamma") or k == "gate" and not gate), k
        assert v is None or not v.any(), k


@gpu
@pytest.mark.parametrize("M", [1, 40, 300])
def test_a_captured_graph_replays_what_the_calls_compute(M):
    """Forwards and backwards in one graph, replayed with other inputs in the same buffers, with eager work between."""
    D, F = 160, 200
    w_in = torch.randint(-2 ** 31, 2 ** 31 - 1, (2 * F, 5), dtype=torch.int32, device=DEV)
    w_out = torch.randint(-2 ** 31, 2 ** 31 - 1, (D, 7), dtype=torch.int32, device=DEV)
    scale = torch.full((2 * F,), 0.08, device=DEV)
    x = torch.empty(M, D, dtype=torch.bfloat16, device=DEV)
    h, y, r, n = (torch.empty(M, c, dtype=torch.bfloat16, device=DEV) for c in (F, D, D, D))
    ws = torch.empty(bnn.gated_bits_backward_workspace(torch.bfloat16, M, F, D), dtype=torch.uint8, device=DEV)

    def work():
        bnn.gated_bits(x, w_in, scale, out=h)
        bnn.linear_bits(h, w_out, scale[:D].clone(), residual=x, out=y)
        bnn.norm_residual(y, x, None, 0.5, bnn.NORM_RMS, None, None, bnn.NORM_LAYER, None, None, 1e-5, M, out=r, out_n=n)
        got = bnn.gated_bits_backward(h, x, w_in, scale, workspace=ws)
        return got["dx"], got["dw"], got["dscale"]

    x.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    for seed in range(4):
        torch.manual_seed(seed)
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in (h, y, r, n, *captured)]
        for t in (h, y, r, n):
            t.zero_()
        eager = work()
        torch.cuda.synchronize()
        for a, b in zip(have, (h, y, r, n, *eager)):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("T", TYPES)
def test_torch_differentiates_the_products(T):
    T = TYPES[T]
    p = Product(20, 48, 70, T, seed=29)
    w_up = torch.cat([p.wd, -p.wd])
    lin = torch.nn.Linear(70, 70).to(DEV, T)
    x = lin(p.xd)
    scale, bias, both = p.scaled.clone().requires_grad_(), p.biased.clone().requires_grad_(), torch.rand(96, device=DEV, requires_grad=True)
    res = torch.randn(20, 48, device=DEV).to(T).requires_grad_()
    y = bnn.linear_bits(x, p.wd, scale, bias, bnn.ACT_GELU, res)
    h = bnn.gated_bits(x, w_up, both, None, bnn.ACT_SILU)
    assert y.requires_grad and h.requires_grad
    dy, dh = torch.randn(20, 48, device=DEV).to(T), torch.randn(20, 48, device=DEV).to(T)
    torch.autograd.backward([y, h], [dy, dh], inputs=[x, scale, bias, res, both, lin.weight])
    a = bnn.linear_bits_backward(dy, x.detach(), p.wd, p.scaled, p.biased, bnn.ACT_GELU)
    b = bnn.gated_bits_backward(dh, x.detach(), w_up, both.detach(), None, bnn.ACT_SILU)
    assert torch.equal(x.grad, a["dx"] + b["dx"])
    assert torch.equal(scale.grad, a["dscale"]) and torch.equal(bias.grad, a["dbias"]) and torch.equal(both.grad, b["dscale"])
    assert torch.equal(res.grad, dy) and lin.weight.grad.any()
    # a gradient that is one number for all; of the scale alone
    s = p.scaled.clone().requires_grad_()
    bnn.linear_bits(p.xd, p.wd, s).sum().backward()
    want = bnn.linear_bits_backward(torch.ones(20, 48, device=DEV).to(T), p.xd, p.wd, p.scaled)["dscale"]
    assert torch.equal(s.grad, want)
    with torch.no_grad():
        assert not bnn.linear_bits(x, p.wd, scale).requires_grad
    assert torch.equal(bnn.linear_bits(x, p.wd, scale, bias, bnn.ACT_GELU, res, out=torch.empty_like(res)), y)
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(bnn.linear_bits(x.detach().requires_grad_(), p.wd).float().square().sum(), both, allow_unused=False)


@gpu
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("rms", "none"), ("none", "rms")])
def test_torch_differentiates_the_norms(post, pre):
    n = Norm(30, 70, 7, torch.float32, post, pre, seed=4)
    leaf = lambda t: None if t is None else t.to(DEV).requires_grad_()
    y, x, gate = leaf(n.y.clone()), leaf(n.x.clone()), leaf(n.gate.clone())
    v = {k: leaf(None if t is None else t.clone()) for k, t in n.vec.items()}

    def call(**kw):
        return bnn.norm_residual(y, x, gate, 0.5, NORMS[post], v["post_gamma"], v["post_beta"], NORMS[pre], v["pre_gamma"], v["pre_beta"],
                                 1e-5, n.R, **kw)

    def check(want):
        for t, k in ((y, "dy"), (x, "dx"), (gate, "dgate"), *((v[k], "d" + k) for k in v)):
            assert (t is None) == (want[k] is None)
            if t is not None:
                assert torch.equal(t.grad, want[k]), k
                t.grad = None

    r, nn = call()
    torch.autograd.backward([r] + ([nn] if nn is not None else []), [n.dr.to(DEV)] + ([n.dn.to(DEV)] if nn is not None else []))
    check(n.back(r.detach().cpu()))
    if pre != "none":                                                  # by one of the results alone
        nothing, nn = call(need_r=False)
        assert nothing is None
        nn.backward(n.dn.to(DEV))
        check(n.back(r.detach().cpu(), dr=False))
        call()[0].backward(n.dr.to(DEV))
        n.dn.zero_()
        check(n.back(r.detach().cpu()))
    out = torch.empty_like(y)
    assert not call(out=out, out_n=torch.empty_like(y) if pre != "none" else None)[0].requires_grad


@gpu
def test_torch_does_not_record_the_block():
    block, x, (w_in, w_out) = small_block()
    block.post_gamma = torch.nn.Parameter(torch.ones(64, device=DEV))
    block.set_weights(w_in.requires_grad_(), w_out)
    x.requires_grad_()
    r, after = block.forward(x, block.first_norm(x), keep=True)
    dx, dn = block.backward(torch.ones_like(r), torch.zeros_like(after))
    assert not any(t.requires_grad for t in (r, after, dx, dn, block.scale_in, *(g for g in block.grads.values() if g is not None)))


# ---- refusals ------------------------------------------------------------------------------------------------------

def test_entry_points_refuse_before_any_launch():
    import ctypes
    lib = bnn.load_library()
    buf = (ctypes.c_uint32 * 64)()
    p = (ctypes.addressof(buf) + 15) // 16 * 16
    INVALID, ALIGN, UNSUPPORTED = 1, 2, 3

    def linear(type=0, x=p, ld_x=40, w=p, ld_w=2, scale=p, bias=p, act=0, res=None, ld_r=0, y=p, ld_y=8, M=2, N=8, K=40):
        return lib.bnn_linear_bits(type, x, ld_x, w, ld_w, scale, bias, act, res, ld_r, y, ld_y, M, N, K, None)

    def gated(type=0, x=p, ld_x=40, w=p, ld_w=2, act=2, h=p, ld_h=8, M=2, F=8, K=40):
        return lib.bnn_gated_bits(type, x, ld_x, w, ld_w, None, None, act, h, ld_h, M, F, K, None)

    for bad in ({"type": 3}, {"type": -1}, {"act": 6}, {"act": -1}, {"M": -1}, {"K": -1}, {"ld_x": 39}, {"ld_w": 1}, {"x": None},
                {"w": None}, {"K": 2 ** 31 - 1, "ld_x": 2 ** 31 - 1, "ld_w": 2 ** 26}, {"M": 2 ** 31}):
        assert linear(**bad) == INVALID and gated(**bad) == INVALID, bad
    for bad in ({"N": -1}, {"ld_y": 7}, {"y": None}, {"res": p, "ld_r": 7}):
        assert linear(**bad) == INVALID, bad
    for bad in ({"F": -1}, {"ld_h": 7}, {"h": None}, {"F": 2 ** 30}):
        assert gated(**bad) == INVALID, bad
    for bad in ({"x": p + 1}, {"w": p + 2}, {"scale": p + 1}, {"bias": p + 2}, {"y": p + 1}, {"res": p + 1, "ld_r": 8},
                {"type": 2, "x": p + 2}, {"type": 2, "y": p + 2}):
        assert linear(**bad) == ALIGN, bad
    assert gated(h=p + 1) == ALIGN
    assert linear(M=2 ** 31 - 10) == UNSUPPORTED
    assert linear(M=0) == 0 and linear(N=0, x=None, w=None) == 0 and gated(F=0) == 0

    def back(dy=p, ld_dy=8, x=p, ld_x=40, dx=p, ld_dx=40, dw=p, ld_dw=40, ds=p, db=p, M=2, N=8, K=40, ws=p, size=None, type=0, act=0):
        need = lib.bnn_linear_bits_backward_workspace(type, M, N, K, act)
        return lib.bnn_linear_bits_backward(type, dy, ld_dy, x, ld_x, p, 2, p, p, act, dx, ld_dx, dw, ld_dw, ds, db, M, N, K, ws,
                                            need if size is None else size, None)

    need = lib.bnn_linear_bits_backward_workspace(0, 2, 8, 40, 0)
    assert need > 0 and need % 16 == 0
    for bad in ({"dy": None}, {"ld_dy": 7}, {"ld_dx": 39}, {"ld_dw": 39}, {"size": need - 1}, {"ws": None}, {"x": None}, {"act": 9}):
        assert back(**bad) == INVALID, bad
    for bad in ({"dy": p + 1}, {"dx": p + 1}, {"dw": p + 1}, {"ds": p + 2}, {"db": p + 2}, {"ws": p + 8}):
        assert back(**bad) == ALIGN, bad
    assert lib.bnn_linear_bits_backward_workspace(5, 2, 8, 40, 0) == -1
    assert lib.bnn_gated_bits_backward_workspace(0, -1, 8, 40, 0) == -1
    assert lib.bnn_gated_bits_backward_workspace(0, 2, 2 ** 31, 40, 0) == -1

    def norm(type=0, y=p, ld_y=8, x=p, ld_x=8, gate=p, ld_g=8, R=1, post=1, pg=p, pb=None, pre=1, qg=p, qb=None, r=p, ld_r=8, n=p,
             ld_n=8, M=2, D=8):
        return lib.bnn_norm_residual(type, y, ld_y, x, ld_x, gate, ld_g, R, 1.0, post, pg, pb, pre, qg, qb, 1e-5, r, ld_r, n, ld_n,
                                     M, D, None)

    for bad in ({"type": 7}, {"post": 3}, {"pre": -1}, {"R": 0}, {"M": -1}, {"D": -1}, {"y": None}, {"n": None}, {"ld_y": 7},
                {"ld_x": 7}, {"ld_g": 7}, {"ld_r": 7}, {"ld_n": 7}, {"pb": p}, {"qb": p}, {"pre": 0, "qg": None}, {"post": 0},
                {"pre": 0, "n": None}):
        assert norm(**bad) == INVALID, bad
    for bad in ({"y": p + 1}, {"n": p + 1}, {"pg": p + 2}, {"qg": p + 1}, {"type": 2, "r": p + 2}):
        assert norm(**bad) == ALIGN, bad
    assert norm(D=16385, ld_y=20000, ld_x=20000, ld_g=20000, ld_r=20000, ld_n=20000) == UNSUPPORTED
    assert norm(M=0) == 0 and norm(D=0) == 0
    assert lib.bnn_norm_residual_backward_workspace(2, 16385, 1) == -1
    assert lib.bnn_norm_residual_backward_workspace(2, 8, 0) == -1


def test_wrappers_refuse_what_the_library_cannot_see():
    x = torch.zeros(2, 40)
    w = torch.zeros(8, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        bnn.linear_bits(x, w)
    with pytest.raises(ValueError, match="device tensor"):
        bnn.norm_residual(x)
    with pytest.raises(ValueError, match="not torch.float64"):
        bnn.linear_bits_backward_workspace(torch.float64, 2, 8, 40)


@gpu
def test_wrappers_check_shapes_types_and_devices():
    x = torch.zeros(2, 40, device=DEV)
    w = torch.zeros(8, 2, dtype=torch.int32, device=DEV)
    vec = torch.zeros(8, device=DEV)
    for bad in ((x.double(), w), (x, w.float()), (x, w[:, :1]), (x.t(), w), (x, w.cpu())):
        with pytest.raises(ValueError):
            bnn.linear_bits(*bad)
    for kw in ({"scale": vec[:7]}, {"scale": vec.half()}, {"bias": vec.cpu()}, {"bias": torch.zeros(16, device=DEV)[::2]},
               {"residual": torch.zeros(2, 7, device=DEV)}, {"residual": torch.zeros(2, 8, device=DEV).half()},
               {"out": torch.zeros(3, 8, device=DEV)}, {"out": torch.zeros(2, 8, device=DEV).bfloat16()}):
        with pytest.raises(ValueError):
            bnn.linear_bits(x, w, **kw)
    with pytest.raises(ValueError):
        bnn.gated_bits(x, w[:7])
    with pytest.raises(bnn.BnnError):
        bnn.gated_bits(x, w, act=17)
    with pytest.raises(ValueError):
        bnn.linear_bits_backward(torch.zeros(2, 7, device=DEV), x, w)
    with pytest.raises(ValueError, match="bytes"):
        bnn.linear_bits_backward(torch.zeros(2, 8, device=DEV), x, w, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        bnn.norm_residual(x, gate=torch.zeros(3, 40, device=DEV), rows_per_gate=2)
    with pytest.raises(ValueError):
        bnn.norm_residual(x, out_n=torch.zeros(2, 40, device=DEV))
    with pytest.raises(ValueError):
        bnn.norm_residual_backward(x, None, x, None, pre=bnn.NORM_RMS)
    with pytest.raises(bnn.BnnError):
        bnn.norm_residual(torch.zeros(1, 16385, device=DEV))
