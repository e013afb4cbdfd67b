"""Quantised activations with packed weights: codes of 8 and 4 bits with scales (quantize_rows, dequantize_rows, norm_residual_q) and
the products that read them (linear_q_bits, gated_q_bits), against their definitions in 64 bits on the CPU.

Codes of stored rows are exact: scales and whole numbers of steps have to be equal.  Where a value is computed before it is
quantised, its error decides which of two codes it gets next to a border: there the result has to be as near to the value as
the nearest code of the scale that was given, and that scale right, both but for the value's own error.  Products: sums of 8-bit
codes are exact, three roundings follow; sums of n products of 4-bit codes in float32 are off by at most (n + 8) 2^-24 of the sum of
magnitudes; activations and the last rounding as for real activations."""
import numpy as np
import pytest
import torch

import paper_1602_02830_amd as bnn
from paper_1602_02830_amd import binding
from test_real_activations import ACTS, DEV, F32, NORMS, ROUND, TINY, TYPES, act_error, close, phi, rounded

gpu = pytest.mark.gpu
KINDS = {"i8": bnn.ROWS_I8, "mx4": bnn.ROWS_MX4}
MX4 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
NAN = float("nan")
INF = float("inf")


# ---- definitions -------------------------------------------------------------------------------------------------

def i8_want(x):
    """(q, s) of float64 rows; s is a float32 by definition."""
    x = x.double()
    most = x.abs().amax(1) if x.shape[1] else torch.zeros(x.shape[0], dtype=torch.float64)
    s = (most.float() / 127).clamp(min=2.0 ** -126).double()
    bad = ~torch.isfinite(x).all(1)
    q = torch.round(x / s[:, None])              # half to even
    q[bad] = 0
    s[bad] = NAN
    return q, s


def blocks_of(x):
    M, K = x.shape
    return torch.nn.functional.pad(x, (0, -K % 32)).reshape(M, (K + 31) // 32, 32)


def mx4_want(x):
    """(c, 2^e) of float64 rows, c in blocks of 32 [M][blocks][32], e [M][blocks]; by trying exponents upwards."""
    b = blocks_of(x.double())
    most = b.abs().amax(2)
    bad = ~torch.isfinite(b).all(2)
    most = torch.where(bad, torch.ones_like(most), most)
    e = torch.full_like(most, -126.0)
    for t in range(-126, 127):
        e = torch.where(most >= 7 * 2.0 ** t, torch.full_like(e, t + 1.0), e)      # 7 * 2^t does not round to 6 * 2^t
    v = b / torch.exp2(e)[:, :, None]
    v = torch.where(bad[:, :, None], torch.zeros_like(v), v)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    c = torch.copysign(torch.round(a / step) * step, v)
    power = torch.exp2(e)
    power[bad] = NAN
    return c, power


def values_of(q):
    """What a QuantizedRows on the GPU holds, decoded on the CPU from its bytes: (codes in blocks [M][blocks][32], scales)."""
    M, K = q.shape
    nb = (K + 31) // 32
    raw = q.codes.cpu().numpy()[:, :nb * (32 if q.kind == bnn.ROWS_I8 else 16)]
    if q.kind == bnn.ROWS_I8:
        by = raw.view(np.int8).reshape(M, nb, 8, 4)                   # byte 4 i + j: element 8 j + i
        c = np.transpose(by, (0, 1, 3, 2)).reshape(M, nb, 32).astype(np.float64)
        return torch.from_numpy(c), q.scales.cpu().double()
    nib = np.stack([raw & 15, raw >> 4], axis=-1).reshape(M, nb, 4, 8)       # nibble 8 i + j: element 4 j + i
    nib = np.transpose(nib, (0, 1, 3, 2)).reshape(M, nb, 32)
    c = MX4[torch.from_numpy((nib & 7).astype(np.int64))] * torch.where(torch.from_numpy(nib & 8) > 0, -1.0, 1.0)
    s = torch.from_numpy(q.scales.cpu().numpy()[:, :nb].astype(np.float64))
    return c, torch.where(s == 255, torch.full_like(s, NAN), torch.exp2(s - 127))


def hat_of(q):
    """x^ in float64 [M][K]."""
    c, s = values_of(q)
    return (c * (s[:, None, None] if q.kind == bnn.ROWS_I8 else s[:, :, None])).reshape(c.shape[0], c.shape[1] * 32)[:, :q.K]


def check_codes(q, x):
    """The codes, scales and pad of quantised stored rows."""
    c, s = values_of(q)
    if q.kind == bnn.ROWS_I8:
        want, ws = i8_want(x)
        want = blocks_of(want)
    else:
        want, ws = mx4_want(x)
        there = torch.isfinite(ws)[:, :, None]
        c, want = torch.where(there, c, 0.0), torch.where(there, want, 0.0)
    assert torch.equal(torch.nan_to_num(s, nan=-1.0), torch.nan_to_num(ws, nan=-1.0)), "scales"
    assert torch.equal(c, want), ("codes", int((c != want).sum()))


def rows_with_borders(M, K, T, seed=0):
    """Rows of many magnitudes with zeros, ties between codes, values that round past the largest code, and sparse large ones."""
    g = torch.Generator().manual_seed(17 * seed + M + 1000 * K)
    x = torch.randn(M, K, generator=g) * torch.exp2(torch.randint(-8, 8, (M, 1), generator=g).float())
    for m in range(M):
        kind = m % 8
        if kind == 1:
            x[m] = 0
        elif kind == 2:                              # half steps of 8 bits, the largest one 127 of them
            x[m] = torch.randint(-254, 255, (K,), generator=g) * 0.25
            x[m, K // 2] = 63.5
        elif kind == 3:                              # borders of 4 bits, under every largest magnitude in a binade
            x[m] = torch.randint(-32, 33, (K,), generator=g) * 0.25
        elif kind == 4:
            x[m] *= (torch.rand(K, generator=g) < 0.05).float() * 30 + 0.01
        elif kind == 5:
            x[m] = 7.0 * torch.sign(x[m])
        elif kind == 6:                              # halves of the largest are 63.5 steps
            x[m] = torch.where(torch.rand(K, generator=g) < 0.5, 0.5, 1.0) * (1 + m / 16)
    return x.to(T)


def placed(t, gap=0, shift=0):
    """Rows `gap` elements apart beyond their length, `shift` elements into a buffer of NaNs."""
    M, K = t.shape
    buf = torch.full((M * (K + gap) + shift + 8,), NAN, dtype=t.dtype, device=DEV)
    v = buf[shift:shift + M * (K + gap)].view(M, K + gap)[:, :K]
    v.copy_(t)
    return v


SIZES = [(1, 1), (3, 7), (5, 31), (2, 32), (9, 33), (40, 100), (17, 512), (9, 513), (33, 1000), (8, 1025), (16, 2047), (9, 4096), (3, 8193), (2, 16384),
         (2, 16385), (8, 20001)]


@gpu
@pytest.mark.parametrize("T", list(TYPES))
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,K", SIZES)
def test_quantise(M, K, kind, T):
    T = TYPES[T]
    x = rows_with_borders(M, K, T)
    q = bnn.quantize_rows(placed(x, 5, 3), KINDS[kind], hat=True)
    check_codes(q, x)
    hat = hat_of(q)
    close(q.hat, hat, ROUND[T] * hat.abs() + TINY[T], "x^")
    if kind == "mx4":
        assert torch.equal(q.hat.cpu().double(), hat)                # a number of each type
    back = bnn.dequantize_rows(q, T)
    assert torch.equal(back, q.hat)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_quantise_random_types_agree(kind):
    """Many rows, walked over by fewer workgroups, and x^ in another type than the rows'."""
    x = rows_with_borders(5000, 96, torch.bfloat16, seed=3)
    q = bnn.quantize_rows(x.to(DEV), KINDS[kind])
    check_codes(q, x)
    again = bnn.quantize_rows(x.float().to(DEV), KINDS[kind])
    assert torch.equal(q.codes, again.codes) and torch.equal(values_of(q)[1], values_of(again)[1])
    for T in TYPES.values():
        hat = hat_of(q)
        close(bnn.dequantize_rows(q, T), hat, ROUND[T] * hat.abs() + TINY[T], "x^")


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("K", [40, 600, 17000])
def test_quantise_special_values(kind, K):
    """Infinities and NaNs make a row (8 bits) or a block (4 bits) NaN and leave the others; the smallest and largest magnitudes."""
    x = torch.randn(12, K, generator=torch.Generator().manual_seed(5))
    x[1, 3], x[2, K - 1], x[3, 35] = NAN, INF, -INF
    x[4] = 0
    x[4, 0] = 2.0 ** -149
    x[5] *= 1e-38
    x[6] *= 2.0 ** -140
    x[7] = x[7].clamp(-1, 1) * 3.4e38
    x[8, 7] = torch.finfo(torch.float32).max
    x[9] = -0.0
    x[10] = 2.0 ** -126 * 127
    q = bnn.quantize_rows(x.to(DEV), KINDS[kind], hat=True)
    check_codes(q, x)
    hat = hat_of(q)
    got = q.hat.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(hat))
    fine = torch.isfinite(hat) & (hat.abs() <= torch.finfo(torch.float32).max)      # what rounds up past the largest float is infinite
    assert torch.isinf(got[torch.isfinite(hat) & ~fine]).all()
    tol = 2.0 ** -24 * hat.abs() + 2.0 ** -150
    assert ((got - hat).abs()[fine] <= tol[fine]).all()


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_quantise_places(kind):
    """x^ in the rows' own place, rows of codes far apart, and nothing written between or behind them."""
    M, K, kind = 19, 333, KINDS[kind]
    x = rows_with_borders(M, K, torch.float16, seed=2)
    want = bnn.quantize_rows(x.to(DEV), kind, hat=True)
    blocks, size = (K + 31) // 32, 32 if kind == bnn.ROWS_I8 else 16
    codes = torch.full((M + 2, blocks * size + 48), 0xA5, dtype=torch.uint8, device=DEV)
    if kind == bnn.ROWS_I8:
        scales = torch.full((M + 2,), 123.0, device=DEV)
        inner = scales[1:-1]
    else:
        scales = torch.full((M + 2, 32), 0xA5, dtype=torch.uint8, device=DEV)
        inner = scales[1:-1, :16]
    real = torch.full((M + 2, K + 9), 7.0, dtype=torch.float16, device=DEV)
    real[1:-1, 1:K + 1] = x.to(DEV)
    place = real[1:-1, 1:K + 1]
    q = bnn.QuantizedRows(kind, K, codes[1:-1, :blocks * size], inner, place)
    assert bnn.quantize_rows(place, kind, out=q) is q
    assert torch.equal(q.codes, want.codes) and torch.equal(place, want.hat)
    assert torch.equal(q.scales if kind == bnn.ROWS_I8 else q.scales[:, :blocks], want.scales if kind == bnn.ROWS_I8 else want.scales[:, :blocks])
    assert (codes[0] == 0xA5).all() and (codes[-1] == 0xA5).all() and (codes[:, blocks * size:] == 0xA5).all()
    edge = scales[[0, -1]]
    assert (edge == (123.0 if kind == bnn.ROWS_I8 else 0xA5)).all()
    if kind == bnn.ROWS_MX4:
        assert (scales[:, blocks:] == 0xA5).all()
    assert (real[0] == 7).all() and (real[-1] == 7).all() and (real[:, 0] == 7).all() and (real[:, K + 1:] == 7).all()


# ---- norms ----------------------------------------------------------------------------------------------------------

def nearest_but_for(q, v, err, what):
    """Quantised values v that are known but for err: scales and codes."""
    c, s = values_of(q)
    if q.kind == bnn.ROWS_I8:
        most, tol = v.abs().amax(1), err.amax(1)
        assert ((s - most / 127).abs() <= tol / 127 + 2.0 ** -23 * s).all(), (what, "scales")
        best = (v / s[:, None] - torch.round(v / s[:, None])).abs() * s[:, None]
        steps = s[:, None]
    else:
        b, e = blocks_of(v), blocks_of(err).amax(2)
        most = b.abs().amax(2)
        assert (most - e < 7 * s).all() and ((most + e >= 3.5 * s) | (s == 2.0 ** -126)).all(), (what, "scales")
        codes = torch.cat([-MX4.flip(0), MX4])
        best = (b[:, :, :, None] - codes * s[:, :, None, None]).abs().amin(3).reshape(v.shape[0], -1)[:, :v.shape[1]]
        steps = s[:, :, None].expand(b.shape).reshape(v.shape[0], -1)[:, :v.shape[1]]
    got = hat_of(q)
    # 2^-20 of a step: what the comparison itself rounds.
    bad = (got - v).abs() > best + 2 * err + 2.0 ** -20 * steps
    assert not bad.any(), (what, int(bad.sum()))


def norm_want(v, kind, gamma, beta, eps):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    v = v * gamma.double() if gamma is not None else v
    return v + beta.double() if beta is not None else v


@gpu
@pytest.mark.parametrize("T", list(TYPES))
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,D,post,pre,gated", [(1, 5, "none", "rms", False), (3, 33, "rms", "rms", True), (40, 100, "layer", "layer", True), (5, 512, "rms", "none", True),
                                                (7, 777, "none", "none", False), (6, 2049, "layer", "rms", True), (300, 96, "rms", "layer", False),
                                                (2, 5000, "rms", "rms", True), (2, 16384, "none", "rms", False)])
def test_norm(M, D, post, pre, gated, kind, T):
    T = TYPES[T]
    g = torch.Generator().manual_seed(M + D)
    y, x = (torch.randn(M, D, generator=g) * 2).to(T), torch.randn(M, D, generator=g).to(T)
    gate = (1 + 0.3 * torch.randn((M + 2) // 3, D, generator=g)).to(T) if gated else None
    vec = {k: (b + 0.3 * torch.randn(D, generator=g)) if side == need or (need is None and side != "none") else None
           for k, side, need, b in (("post_gamma", post, None, 1), ("post_beta", post, "layer", 0), ("pre_gamma", pre, None, 1), ("pre_beta", pre, "layer", 0))}
    on = {k: v.to(DEV) if v is not None else None for k, v in vec.items()}
    gd = gate.to(DEV) if gated else None
    args = (placed(y, 3, 1), placed(x, 0, 5), gd, 0.75, NORMS[post], on["post_gamma"], on["post_beta"], NORMS[pre], on["pre_gamma"], on["pre_beta"], 1e-5, 3)
    r, q = bnn.norm_residual_q(*args, KINDS[kind], hat=True)
    real_r, real_n = bnn.norm_residual(*args)
    assert torch.equal(r, real_r)
    t = norm_want(y.double(), post, vec["post_gamma"], vec["post_beta"], 1e-5) * 0.75
    if gated:
        t = t * gate.double().repeat_interleave(3, 0)[:M]
    r64 = x.double() + t
    n64 = norm_want(r64, pre, vec["pre_gamma"], vec["pre_beta"], 1e-5)
    # A norm's result is off by (D + 16) 2^-24 of the row's largest magnitude (the statistics' relative errors, and a few roundings),
    # two norms by twice that, scaled by the second one's growth.
    grow = (n64.abs().amax(1, keepdim=True) + 1) / r64.abs().amax(1, keepdim=True).clamp(min=1e-3)
    err = (D + 16) * F32 * (n64.abs().amax(1, keepdim=True) + 2 * grow * (r64.abs().amax(1, keepdim=True) + y.double().abs().amax(1, keepdim=True)))
    nearest_but_for(q, n64, err.expand_as(n64).contiguous(), "n^")
    hat = hat_of(q)
    close(q.hat, hat, ROUND[T] * hat.abs() + TINY[T], "n^ as reals")
    # Without r, without n^, and into places that are there.
    _, only = bnn.norm_residual_q(*args, KINDS[kind], need_r=False)
    assert only.hat is None and torch.equal(only.codes, q.codes)
    out, out_q = torch.empty_like(r), bnn.quantized_rows(M, D, KINDS[kind], DEV, T)
    got = bnn.norm_residual_q(*args, KINDS[kind], out=out, out_q=out_q)
    assert got[0] is out and got[1] is out_q and torch.equal(out, r) and torch.equal(out_q.codes, q.codes) and torch.equal(out_q.hat, q.hat)


# ---- products -------------------------------------------------------------------------------------------------------

class QProduct:
    """Quantised rows on the GPU, with the values that they hold in 64 bits; weights have junk in pad bits and pad words."""

    def __init__(self, M, N, K, kind, T, scale=True, bias=True, gap=0, seed=0):
        g = torch.Generator().manual_seed(1000 * seed + M + 7 * N + 31 * K)
        self.T, self.kind = T, KINDS[kind]
        x = torch.randn(M, K, generator=g) * (1 + 15 * (torch.rand(K, generator=g) < 0.02).float())
        x[M // 2:M // 2 + 1] *= 2.0 ** -9
        self.q = bnn.quantize_rows(x.to(DEV), self.kind, hat=False)
        if gap:
            codes = torch.full((M, self.q.codes.shape[1] + 16 * gap), 0xFF, dtype=torch.uint8, device=DEV)
            codes[:, :self.q.codes.shape[1]] = self.q.codes
            self.q.codes = codes[:, :self.q.codes.shape[1]]
            if self.kind == bnn.ROWS_MX4:
                wide = self.q.scales.shape[1]
                scales = torch.full((M, wide + 16 * gap), 0xFF, dtype=torch.uint8, device=DEV)
                scales[:, :(K + 31) // 32] = self.q.scales[:, :(K + 31) // 32]         # the bytes past K's blocks: NaN, not to be read as scales
                self.q.scales = scales[:, :wide]
        self.x = hat_of(self.q)
        self.w = torch.randint(0, 2, (N, K), generator=g).mul_(2).sub_(1).double()
        self.scale = (torch.rand(N, generator=g) + 0.5) / max(K, 1) ** 0.5 if scale else None
        self.bias = 0.3 * torch.randn(N, generator=g) if bias else None
        words = (K + 31) // 32
        bits = np.zeros((N, words * 32), np.uint8)
        bits[:, :K] = self.w.numpy() > 0
        bits[:, K:] = 1
        packed = np.packbits(bits, axis=1, bitorder="little").view(np.uint32).reshape(N, words)
        buf = np.full((N, words + (3 if gap else 0)), 0x5A5A5A5A, np.uint32)
        buf[:, :words] = packed
        self.wd = torch.tensor(buf.view(np.int32), device=DEV)[:, :words] if N else torch.empty((0, words), dtype=torch.int32, device=DEV)
        self.scaled = self.scale.to(DEV) if scale else None
        self.biased = self.bias.to(DEV) if bias else None

    def z(self):
        """z and a bound of its error."""
        s = self.x @ self.w.t()
        a = self.scale.double() if self.scale is not None else torch.ones(self.w.shape[0], dtype=torch.float64)
        b = self.bias.double() if self.bias is not None else torch.zeros(self.w.shape[0], dtype=torch.float64)
        z = s * a + b
        # 8 bits: the sum is exact; to float, times the row's scale, times the channel's and bias in one.
        es = 2 * F32 * s.abs() if self.kind == bnn.ROWS_I8 else (self.x.shape[1] + 8) * F32 * self.x.abs().sum(1, keepdim=True).expand_as(s)
        return z, 1.01 * es * a + F32 * (z.abs() + es * a)


def result(p, act, gated=False, residual=None):
    """The result in 64 bits, and a bound of its error before the last rounding."""
    z, ez = p.z()
    if not gated:
        f, ef = phi(z, act)[0], act_error(z, ez, act)[0]
        if residual is not None:
            f = f + residual.double()
            ef = ef + F32 * (f.abs() + ef)
        return f, ef
    F = z.shape[1] // 2
    zg, zu, eg, eu = z[:, :F], z[:, F:], ez[:, :F], ez[:, F:]
    f, ef = phi(zg, act)[0], act_error(zg, eg, act)[0]
    h = f * zu
    return h, (f.abs() + ef) * eu + ef * zu.abs() + F32 * (h.abs() + ef * zu.abs() + f.abs() * eu + ef * eu)


PRODUCTS = [(1, 1, 1), (1, 64, 32), (3, 17, 40), (16, 48, 512), (2, 33, 513), (5, 100, 1030), (17, 96, 4096), (8, 40, 8200), (33, 130, 700), (70, 257, 333), (130, 520, 1024),
            (300, 300, 96), (257, 300, 128), (100, 260, 256), (70, 70, 384), (65, 96, 512), (300, 136, 640), (90, 520, 1152), (513, 200, 896), (66, 64, 4224), (130, 70, 97), (80, 130, 130), (68, 40, 2050), (129, 300, 3333), (66, 33, 545)]


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_linear(M, N, K, kind):
    for T, act, scale, bias, res in ((torch.bfloat16, "none", True, True, True), (torch.float32, "gelu", True, False, False), (torch.float16, "silu", True, True, False),
                                     (torch.float32, "none", False, False, True)):
        p = QProduct(M, N, K, kind, T, scale, bias, gap=1 if T == torch.float16 else 0)
        r = torch.randn(M, N, generator=torch.Generator().manual_seed(1)).to(T) if res else None
        want, err = result(p, act, residual=r)
        y = bnn.linear_q_bits(p.q, p.wd, p.scaled, p.biased, ACTS[act], placed(r, 3, 1) if res else None, T)
        close(y, want, rounded(want, err, T), "y")
        if res:                                                 # in the residual's place
            place = r.to(DEV)
            assert bnn.linear_q_bits(p.q, p.wd, p.scaled, p.biased, ACTS[act], place, out=place) is place
            assert torch.equal(place, y)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,F,K", PRODUCTS)
def test_gated(M, F, K, kind):
    for T, act, scale, bias in ((torch.bfloat16, "silu", True, False), (torch.float32, "gelu_tanh", True, True), (torch.float16, "sigmoid", True, True)):
        p = QProduct(M, 2 * F, K, kind, T, scale, bias, gap=1 if T == torch.float16 else 0)
        want, err = result(p, act, gated=True)
        h = bnn.gated_q_bits(p.q, p.wd, p.scaled, p.biased, ACTS[act], T)
        close(h, want, rounded(want, err, T), "h")
        # Quantised for the product that follows, with and without h^.
        q = bnn.gated_q_bits(p.q, p.wd, p.scaled, p.biased, ACTS[act], T, out_kind=bnn.ROWS_MX4, hat=True)
        nearest_but_for(q, want, err, "h^")
        c, _ = values_of(q)
        assert (c.reshape(M, -1)[:, F:] == 0).all()
        assert torch.equal(q.hat, bnn.dequantize_rows(q, T))
        only = bnn.gated_q_bits(p.q, p.wd, p.scaled, p.biased, ACTS[act], T, out_q=bnn.quantized_rows(M, F, bnn.ROWS_MX4, DEV))
        assert only.hat is None and torch.equal(only.codes, q.codes) and torch.equal(only.scales[:, :(F + 31) // 32], q.scales[:, :(F + 31) // 32])


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_products_of_nothing(kind):
    """No elements of K: the bias alone, whatever the scales are; no rows, no channels."""
    p = QProduct(4, 40, 0, kind, torch.float32)
    if kind == "i8":
        p.q.scales.fill_(NAN)
    y = bnn.linear_q_bits(p.q, p.wd, p.scaled, p.biased, ACTS["relu"], dtype=torch.float32)
    assert torch.equal(y.cpu(), p.bias.clamp(min=0).expand(4, 40))
    for M, N, K in ((0, 32, 64), (4, 0, 64)):
        p = QProduct(M, N, K, kind, torch.bfloat16)
        assert bnn.linear_q_bits(p.q, p.wd, p.scaled, p.biased).shape == (M, N)
        assert bnn.gated_q_bits(p.q, p.wd, p.scaled, p.biased).shape == (M, N // 2)
        q = bnn.gated_q_bits(p.q, p.wd, p.scaled, p.biased, out_kind=bnn.ROWS_MX4)
        assert q.shape == (M, N // 2)
    assert bnn.quantize_rows(torch.empty(0, 5, device=DEV), KINDS[kind]).shape == (0, 5)


@gpu
def test_scales_of_rows_of_nothing():
    """The least one, from quantisation and from the norm alike; MX4 rows of nothing have no block."""
    x = torch.empty(5, 0, device=DEV)
    for give in (lambda q: bnn.quantize_rows(x, out=q), lambda q: bnn.norm_residual_q(x, pre=bnn.NORM_RMS, out_q=q, need_r=False)):
        q = bnn.quantized_rows(5, 0, bnn.ROWS_I8, DEV)
        q.scales.fill_(NAN)
        give(q)
        assert torch.equal(q.scales.cpu(), torch.full((5,), 2.0 ** -126))
    assert bnn.norm_residual_q(x, pre=bnn.NORM_RMS, kind=bnn.ROWS_MX4, need_r=False)[1].shape == (5, 0)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_products_of_nan_rows(kind):
    """A row (8 bits) or block (4 bits) that stands for NaN makes its own row of the result NaN, no other."""
    x = torch.randn(20, 300, device=DEV)
    x[3, 77], x[19, 299] = NAN, INF
    w = bnn.pack_sign(torch.randn(64, 300, device=DEV))
    q = bnn.quantize_rows(x, KINDS[kind])
    y = bnn.linear_q_bits(q, w)
    bad = torch.isnan(y).all(1)
    assert bad[[3, 19]].all() and int(torch.isnan(y).any(1).sum()) == 2
    h = bnn.gated_q_bits(q, w, out_kind=bnn.ROWS_MX4, hat=True)
    assert torch.isnan(h.hat).any(1).nonzero().flatten().tolist() == [3, 19]


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_more_rows_than_a_grid_has_places(kind):
    """Small tiles of more than 65535 times 16 rows: of no elements, and of one block, where the sums are exact."""
    M = 65535 * 16 + 37
    q = bnn.quantize_rows(torch.empty(M, 0, device=DEV), KINDS[kind])
    bias = torch.randn(20, device=DEV)
    y = bnn.linear_q_bits(q, torch.empty(20, 0, dtype=torch.int32, device=DEV), None, bias, dtype=torch.float32)
    assert torch.equal(y, bias.expand(M, 20))
    x = torch.randint(-7, 8, (M, 32), device=DEV).float()
    x[:, 0] = 127 if kind == "i8" else 6                   # steps of 1; halves are not asked for
    w = bnn.pack_sign(torch.randn(9, 32, device=DEV))
    q = bnn.quantize_rows(x, KINDS[kind], hat=True)
    assert torch.equal(bnn.linear_q_bits(q, w, dtype=torch.float32), bnn.linear_bits(q.hat, w))
    h = bnn.gated_q_bits(q, w[:8], dtype=torch.float32)
    assert torch.equal(h[-100:], bnn.gated_q_bits(bnn.quantize_rows(x[-100:], KINDS[kind]), w[:8], dtype=torch.float32))


@gpu
def test_longest_rows_of_8_bits():
    """The largest sums that 32 bits hold: every product 127."""
    K = 1 << 18
    q = bnn.quantize_rows(torch.ones(2, K, device=DEV), bnn.ROWS_I8)
    w = torch.full((3, K // 32), -1, dtype=torch.int32, device=DEV)
    w[1] = 0
    w[2, ::2] = 0
    y = bnn.linear_q_bits(q, w, dtype=torch.float32).cpu().double()
    s = float(q.scales[0].cpu().double()) * 127
    assert ((y - torch.tensor([s * K, -s * K, 0.0])).abs() <= 2.0 ** -22 * K).all()
    with pytest.raises(bnn.BnnError) as e:
        bnn.linear_q_bits(bnn.quantize_rows(torch.ones(1, K + 1, device=DEV), bnn.ROWS_I8), torch.zeros(3, K // 32 + 1, dtype=torch.int32, device=DEV))
    assert e.value.status == 3


# ---- calls ------------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_wrappers_and_native_calls_agree(kind, monkeypatch):
    p = QProduct(9, 64, 130, kind, torch.bfloat16)
    x = torch.randn(9, 130, device=DEV).bfloat16()

    def calls():
        q = bnn.quantize_rows(x, p.kind, out=bnn.quantized_rows(9, 130, p.kind, DEV, torch.bfloat16))
        r, n = bnn.norm_residual_q(x, x, None, 0.5, pre=bnn.NORM_RMS, kind=p.kind, out=torch.empty_like(x),
                                   out_q=bnn.quantized_rows(9, 130, p.kind, DEV, torch.bfloat16))
        y = bnn.linear_q_bits(q, p.wd, p.scaled, p.biased, out=torch.empty(9, 64, dtype=torch.float16, device=DEV))
        h = bnn.gated_q_bits(n, p.wd, p.scaled, p.biased, out=torch.empty(9, 32, device=DEV))
        hq = bnn.gated_q_bits(n, p.wd, p.scaled, p.biased, out_q=bnn.quantized_rows(9, 32, bnn.ROWS_MX4, DEV, torch.float32))
        back = bnn.dequantize_rows(n, out=torch.empty(9, 130, device=DEV))
        return [q.codes, q.hat, r, n.codes, n.hat, y, h, hq.codes, hq.hat, back]

    bnn.load_library()
    native = calls()
    monkeypatch.setattr(binding, "_calls", None)
    for a, b in zip(native, calls()):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_another_stream_and_a_graph(kind):
    """A run of the operators, as they are used, on another stream and captured; replays with new inputs, eager work between them."""
    kind = KINDS[kind]
    M, D, F = 40, 256, 320
    g = torch.Generator(device=DEV).manual_seed(3)
    w_in, w_out = bnn.pack_sign(torch.randn(2 * F, D, device=DEV, generator=g)), bnn.pack_sign(torch.randn(D, F, device=DEV, generator=g))
    scale_in, scale_out = torch.rand(2 * F, device=DEV, generator=g) / 16, torch.rand(D, device=DEV, generator=g) / 16
    x = torch.randn(M, D, device=DEV, generator=g).bfloat16()
    n, n2, h = (bnn.quantized_rows(M, c, kind, DEV) for c in (D, D, F))
    r0, r, y, hr = (torch.empty(M, c, dtype=torch.bfloat16, device=DEV) for c in (D, D, D, F))

    def block():
        bnn.norm_residual_q(x, pre=bnn.NORM_RMS, kind=kind, out=r0, out_q=n)
        if kind == bnn.ROWS_MX4:
            bnn.gated_q_bits(n, w_in, scale_in, out_q=h)
        else:
            bnn.quantize_rows(bnn.gated_q_bits(n, w_in, scale_in, out=hr), kind, out=h)
        bnn.linear_q_bits(h, w_out, scale_out, out=y)
        bnn.norm_residual_q(y, x, pre=bnn.NORM_RMS, kind=kind, out=r, out_q=n2)

    def outcome():
        return [t.clone() for t in (r, n2.codes, y)]

    block()
    torch.cuda.synchronize()
    eager = outcome()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for t in (r, n2.codes, y):
            t.zero_()
        block()
    side.synchronize()
    for a, b in zip(eager, outcome()):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for i in range(4):
        x.copy_(torch.randn(M, D, device=DEV, generator=g).bfloat16())
        block()
        torch.cuda.synchronize()
        eager = outcome()
        r.zero_()
        n2.codes.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, outcome()):
            assert torch.equal(a, b), i


def test_refusals(monkeypatch):
    """Sizes, kinds, types and alignment that the library refuses, before it looks at memory."""
    lib = bnn.load_library()
    at = 1 << 20                      # never read

    def quantise(rows=0, type=0, x=at, ld_x=64, codes=at, ld_c=64, scales=at, ld_s=16, hat=0, ld_h=64, M=2, K=64):
        return lib.bnn_quantize_rows(rows, type, x, ld_x, codes, ld_c, scales, ld_s, hat, ld_h, M, K, 0)

    for bad in (dict(rows=2), dict(rows=-1), dict(type=3), dict(M=-1), dict(K=-1), dict(ld_x=63), dict(ld_c=48), dict(rows=1, ld_c=16), dict(rows=1, ld_s=0, K=33),
                dict(x=0), dict(codes=0), dict(scales=0), dict(hat=at, ld_h=63), dict(K=1 << 31)):
        assert quantise(**bad) == 1, bad
    for bad in (dict(x=at + 1), dict(codes=at + 8), dict(ld_c=72), dict(scales=at + 2), dict(rows=1, ld_s=24), dict(rows=1, scales=at + 8, ld_s=16), dict(hat=at + 1), dict(type=2, hat=at + 2)):
        assert quantise(**bad) == 2, bad
    assert quantise(M=0) == 0

    def dequantise(rows=0, type=0, codes=at, ld_c=64, scales=at, ld_s=4, x=at, ld_x=64, M=2, K=64):
        return lib.bnn_dequantize_rows(rows, type, codes, ld_c, scales, ld_s, x, ld_x, M, K, 0)

    for bad in (dict(rows=5), dict(type=-1), dict(ld_x=63), dict(ld_c=32), dict(codes=0), dict(scales=0), dict(x=0)):
        assert dequantise(**bad) == 1, bad
    assert dequantise(x=at + 1) == 2 and dequantise(K=0) == 0

    def norm(type=0, rows=0, codes=at, ld_c=64, scales=at, ld_s=4, hat=0, pre=1, gamma=0, post_gamma=0, y=at, D=64, per=1, M=2):
        return lib.bnn_norm_residual_q(type, y, D, None, 0, None, 0, per, 1.0, 0, post_gamma, None, pre, gamma, None, 1e-5, None, 0, rows, codes, ld_c,
                                       scales, ld_s, hat, D, M, D, 0)

    for bad in (dict(type=7), dict(rows=3), dict(codes=0), dict(scales=0), dict(ld_c=32), dict(pre=3), dict(pre=0, gamma=at), dict(post_gamma=at), dict(y=0), dict(per=0)):
        assert norm(**bad) == 1, bad
    assert norm(D=16385, ld_c=1 << 16) == 3 and norm(codes=at + 4) == 2 and norm(hat=at + 1) == 2 and norm(M=0) == 0

    def linear(rows=0, codes=at, ld_c=64, scales=at, ld_s=4, w=at, ld_w=2, scale=0, act=0, type=0, residual=0, ld_r=8, y=at, ld_y=8, M=2, N=8, K=64):
        return lib.bnn_linear_q_bits(rows, codes, ld_c, scales, ld_s, w, ld_w, scale, None, act, type, residual, ld_r, y, ld_y, M, N, K, 0)

    for bad in (dict(rows=2), dict(act=6), dict(type=3), dict(ld_w=1), dict(ld_y=7), dict(residual=at, ld_r=7), dict(codes=0), dict(w=0), dict(y=0), dict(ld_c=32),
                dict(rows=1, ld_c=16), dict(M=-1), dict(N=-1), dict(K=-1), dict(scales=0)):
        assert linear(**bad) == 1, bad
    for bad in (dict(codes=at + 8), dict(w=at + 2), dict(scale=at + 1), dict(y=at + 1), dict(residual=at + 1), dict(ld_c=72), dict(scales=at + 1)):
        assert linear(**bad) == 2, bad
    big = 1 << 18
    assert linear(K=big + 1, ld_c=2 * big, ld_w=big) == 3
    assert linear(M=0) == 0 and linear(N=0) == 0

    def gated(rows=1, h=at, ld_h=8, oc=0, ld_oc=16, os=0, ld_os=16, F=8, M=2, K=64):
        return lib.bnn_gated_q_bits(rows, at, 64, at, 16, at, 2, None, None, 2, 0, h, ld_h, oc, ld_oc, os, ld_os, M, F, K, 0)

    for bad in (dict(h=0), dict(ld_h=7), dict(oc=at), dict(os=at), dict(oc=at, os=at, ld_oc=0), dict(oc=at, os=at, ld_os=0), dict(F=-1), dict(F=1 << 30)):
        assert gated(**bad) == 1, bad
    assert gated(oc=at + 4, os=at) == 2 and gated(h=at + 1) == 2 and gated(M=0) == 0


@gpu
def test_refusals_of_the_wrappers():
    x = torch.randn(4, 64, device=DEV)
    w = bnn.pack_sign(torch.randn(8, 64, device=DEV))
    q = bnn.quantize_rows(x, bnn.ROWS_MX4)
    R = bnn.QuantizedRows

    def refuses(f, error=ValueError):
        with pytest.raises(error):
            f()

    refuses(lambda: bnn.quantize_rows(x.double()))
    refuses(lambda: bnn.quantize_rows(x.cpu()))
    refuses(lambda: bnn.quantize_rows(x, 2))
    refuses(lambda: bnn.quantize_rows(x, out=bnn.quantized_rows(4, 65, bnn.ROWS_I8, DEV)))
    refuses(lambda: bnn.quantize_rows(x, out=bnn.quantized_rows(3, 64, bnn.ROWS_MX4, DEV)))
    refuses(lambda: bnn.quantize_rows(x, out=bnn.quantized_rows(4, 64, bnn.ROWS_I8, DEV, torch.bfloat16)))
    refuses(lambda: bnn.quantized_rows(-1, 4))
    refuses(lambda: bnn.dequantize_rows(q, torch.float64))
    refuses(lambda: bnn.dequantize_rows(q, out=torch.empty(4, 63, device=DEV)))
    refuses(lambda: bnn.dequantize_rows(R(bnn.ROWS_I8, 64, q.codes, q.scales)))
    refuses(lambda: bnn.dequantize_rows(x))
    refuses(lambda: bnn.linear_q_bits(x, w))
    refuses(lambda: bnn.linear_q_bits(x, w, out=torch.empty(4, 8, device=DEV)))
    refuses(lambda: bnn.linear_q_bits(q, w[:, :1]))
    refuses(lambda: bnn.linear_q_bits(q, w, out=torch.empty(4, 9, device=DEV)))
    refuses(lambda: bnn.linear_q_bits(q, w, torch.ones(9, device=DEV)))
    refuses(lambda: bnn.linear_q_bits(q, w, residual=torch.empty(4, 8, device=DEV), out=torch.empty(4, 8, device=DEV).half()))
    refuses(lambda: bnn.linear_q_bits(q, w, act=9), bnn.BnnError)
    refuses(lambda: bnn.linear_q_bits(R(q.kind, 64, q.codes[:3], q.scales), w))
    refuses(lambda: bnn.linear_q_bits(R(q.kind, 64, q.codes[:, :16], q.scales), w))
    refuses(lambda: bnn.linear_q_bits(R(q.kind, 64, q.codes, q.scales[:, :2]), w))
    refuses(lambda: bnn.gated_q_bits(q, w[:7]))
    refuses(lambda: bnn.gated_q_bits(q, w, out_kind=bnn.ROWS_I8))
    refuses(lambda: bnn.gated_q_bits(q, w, out_q=bnn.quantized_rows(4, 4, bnn.ROWS_I8, DEV)))
    refuses(lambda: bnn.gated_q_bits(q, w, out=torch.empty(4, 4, device=DEV), out_kind=bnn.ROWS_MX4))
    refuses(lambda: bnn.gated_q_bits(q, w, out_q=bnn.quantized_rows(4, 5, bnn.ROWS_MX4, DEV)))
    refuses(lambda: bnn.norm_residual_q(x, out_q=bnn.quantized_rows(4, 32, bnn.ROWS_I8, DEV)))
    refuses(lambda: bnn.norm_residual_q(x, x[:3], pre=bnn.NORM_RMS))


@pytest.mark.parametrize("native", [True, False])
def test_what_is_no_rows_is_refused(native, monkeypatch):
    """As any other argument: by a ValueError, before the GPU or a native call sees it."""
    if not native:
        monkeypatch.setattr(binding, "_calls", None)
    x, w, q = torch.zeros(4, 64), torch.zeros(8, 2, dtype=torch.int32), bnn.quantized_rows(4, 64, bnn.ROWS_MX4, "cpu")
    for bad in (lambda: bnn.quantize_rows(x, out=x), lambda: bnn.quantize_rows(torch.zeros(4, requires_grad=True)),
                lambda: bnn.norm_residual_q(x, out_q=x), lambda: bnn.norm_residual_q(x, out=x, out_q=x), lambda: bnn.gated_q_bits(q, w, out_q=x),
                lambda: bnn.gated_q_bits(q, w, out_kind=bnn.ROWS_I8, out_q=q)):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("native", [True, False])
def test_another_kind_than_that_of_given_rows_is_refused(native, monkeypatch):
    """Before anything is written.  Rows that are given without a kind beside them keep theirs."""
    class Calls:
        quantize_rows = norm_residual_q = staticmethod(lambda *a: 0)

    monkeypatch.setattr(binding, "_calls", Calls if native else None)
    x = torch.zeros(4, 64)
    for kind, other in ((bnn.ROWS_I8, bnn.ROWS_MX4), (bnn.ROWS_MX4, bnn.ROWS_I8)):
        q = bnn.quantized_rows(4, 64, kind, "cpu")
        for bad in (lambda: bnn.quantize_rows(x, other, out=q), lambda: bnn.norm_residual_q(x, kind=other, out=x, out_q=q),
                    lambda: bnn.norm_residual_q(x, kind=other, out_q=q)):
            with pytest.raises(ValueError, match="kind"):
                bad()
        if native:
            for fine in (None, kind):
                assert bnn.quantize_rows(x, fine, out=q) is q and bnn.norm_residual_q(x, kind=fine, out=x, out_q=q)[1] is q
            assert bnn.quantize_rows(x, out=q) is q and bnn.norm_residual_q(x, out=x, out_q=q)[1] is q


@pytest.mark.parametrize("native", [True, False])
def test_given_rows_without_a_place_for_the_values_asked_for_are_refused(native, monkeypatch):
    """hat=True with rows that have no hat: by a ValueError, before anything is written."""
    class Calls:
        quantize_rows = norm_residual_q = gated_q_bits_rows = staticmethod(lambda *a: 0)

    monkeypatch.setattr(binding, "_calls", Calls if native else None)
    x, w = torch.zeros(4, 64), torch.zeros(128, 2, dtype=torch.int32)
    n = bnn.quantized_rows(4, 64, bnn.ROWS_I8, "cpu")
    calls = {"quantise": lambda q, hat: bnn.quantize_rows(x, hat=hat, out=q), "norm": lambda q, hat: bnn.norm_residual_q(x, out=x, out_q=q, hat=hat)[1],
             "norm alone": lambda q, hat: bnn.norm_residual_q(x, out_q=q, need_r=False, hat=hat)[1],
             "gated": lambda q, hat: bnn.gated_q_bits(n, w, out_q=q, hat=hat),
             "gated, kind": lambda q, hat: bnn.gated_q_bits(n, w, out_kind=q.kind, out_q=q, hat=hat)}
    for name, call in calls.items():
        without, with_hat = (bnn.quantized_rows(4, 64, bnn.ROWS_MX4, "cpu", T) for T in (None, torch.float32))
        with pytest.raises(ValueError, match="hat"):
            call(without, True)
        if native and name in ("quantise", "norm", "gated"):
            assert call(without, False) is without and call(with_hat, True) is with_hat and call(with_hat, False) is with_hat


def test_the_type_of_a_quantised_result_reaches_the_library(monkeypatch):
    """Activations are as accurate as the result's type asks: that of h^, else `dtype`, else of x^, else bfloat16; by the native call
    path as by the other."""
    got = []

    class Calls:
        @staticmethod
        def gated_q_bits_rows(*a):
            got.append(a[-1])
            return 0

    monkeypatch.setattr(binding, "_calls", Calls)
    types = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
    w = torch.zeros(8, 2, dtype=torch.int32)
    for x_type in (None, torch.float16):
        for dtype in (None, torch.float32):
            for hat in (None, torch.bfloat16):
                x, out = bnn.quantized_rows(4, 64, bnn.ROWS_I8, "cpu", x_type), bnn.quantized_rows(4, 4, bnn.ROWS_MX4, "cpu", hat)
                assert bnn.gated_q_bits(x, w, dtype=dtype, out_q=out) is out
                assert got.pop() == types[hat or dtype or x_type or torch.bfloat16]


@pytest.mark.parametrize("T", list(TYPES))
@pytest.mark.parametrize("kind", list(KINDS))
def test_the_type_of_the_blocks_stream_reaches_the_library(kind, T, monkeypatch):
    """The block's activations are as accurate as its stream: its gated product gets the stream's type, whether its result is quantised
    there (4 bits) or written out (8)."""
    got = []

    class Calls:
        @staticmethod
        def gated_q_bits_rows(*a):
            got.append(a[-1])
            return 0

        @staticmethod
        def gated_q_bits(*a):
            got.append(binding._TYPES[a[-1].dtype])
            return 0

    for name in ("quantize_rows", "linear_q_bits", "norm_residual_q"):
        setattr(Calls, name, staticmethod(lambda *a: 0))
    monkeypatch.setattr(binding, "_calls", Calls)
    monkeypatch.setattr(binding, "pack_sign", lambda w: torch.zeros(w.shape[0], (w.shape[1] + 31) // 32, dtype=torch.int32))
    block = bnn.BinaryFeedForward(torch.randn(2 * 40, 64), torch.randn(64, 40), rows=KINDS[kind])
    block.forward(torch.zeros(3, 64, dtype=TYPES[T]), bnn.quantized_rows(3, 64, KINDS[kind], "cpu"))
    assert got == [binding._TYPES[TYPES[T]]]


# ---- differentiation ---------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_torch_differentiates_straight_through(kind):
    """A norm, the gated product, the quantisation of its result and the second product, recorded: gradients are those of the same
    calls on real rows at the values that the codes stand for."""
    kind = KINDS[kind]
    M, D, F = 24, 96, 70
    g = torch.Generator(device=DEV).manual_seed(11)

    def leaf(*shape, std=1.0):
        return (torch.randn(*shape, device=DEV, generator=g) * std).requires_grad_()

    x, gamma, s_in, s_out, bias = leaf(M, D), leaf(D), leaf(2 * F, std=0.1), leaf(D, std=0.1), leaf(2 * F)
    w_in, w_out = bnn.pack_sign(torch.randn(2 * F, D, device=DEV, generator=g)), bnn.pack_sign(torch.randn(D, F, device=DEV, generator=g))
    up = torch.randn(M, D, device=DEV, generator=g)
    leaves = (x, gamma, s_in, s_out, bias)

    r, n = bnn.norm_residual_q(x, pre=bnn.NORM_RMS, pre_gamma=gamma, kind=kind)
    assert n.hat.requires_grad and not n.codes.requires_grad
    if kind == bnn.ROWS_MX4:
        h = bnn.gated_q_bits(n, w_in, s_in, bias, out_kind=kind)
    else:
        h = bnn.quantize_rows(bnn.gated_q_bits(n, w_in, s_in, bias), kind)
    y = bnn.linear_q_bits(h, w_out, s_out, residual=r)
    got = torch.autograd.grad(y, leaves, up)

    # The same by hand, from the backward calls on real rows.
    with torch.no_grad():
        two = bnn.linear_bits_backward(up, h.hat, w_out, s_out)
        one = bnn.gated_bits_backward(two["dx"], n.hat, w_in, s_in, bias)
        first = bnn.norm_residual_backward(up, one["dx"], x, r, pre=bnn.NORM_RMS, pre_gamma=gamma)
    for a, b, name in zip(got, (first["dy"], first["dpre_gamma"], one["dscale"], two["dscale"], one["dbias"]), ("x", "gamma", "s_in", "s_out", "bias")):
        assert torch.equal(a, b), name
    # Against differences, where the function is smooth: the channels' scales of the second product.
    with torch.no_grad():
        step = 2.0 ** -6
        d = torch.randn(D, device=DEV, generator=g)
        at = lambda t: bnn.linear_q_bits(h, w_out, (s_out + t * d).detach(), residual=r.detach()).double()
        slope = float(((at(step) - at(-step)) / (2 * step) * up.double()).sum())
        want = float((got[3].double() * d.double()).sum())
        size = float((h.hat.double().abs().sum(1, keepdim=True) * up.double().abs() * d.double().abs()).sum())
    assert abs(slope - want) <= 2.0 ** -24 * 64 / step * size       # linear in the scales: rounding alone


@gpu
def test_gradients_need_matching_types_and_kept_values():
    x = torch.randn(4, 64, device=DEV, requires_grad=True)
    w = bnn.pack_sign(torch.randn(8, 64, device=DEV))
    q = bnn.quantize_rows(x, bnn.ROWS_MX4)
    with pytest.raises(ValueError):
        bnn.linear_q_bits(q, w, dtype=torch.bfloat16)
    y = bnn.linear_q_bits(q, w)
    assert y.dtype == torch.float32 and y.requires_grad
    # Without x^, the scale's gradient comes from the codes.
    s = torch.ones(8, device=DEV, requires_grad=True)
    plain = bnn.quantize_rows(x.detach(), bnn.ROWS_MX4)
    (ds,) = torch.autograd.grad(bnn.linear_q_bits(plain, w, s, dtype=torch.float32).sum(), s)
    want = hat_of(plain) @ torch.where(torch.from_numpy(np.unpackbits(w.cpu().numpy().view(np.uint8), axis=1, bitorder="little")) > 0, 1.0, -1.0).double().t()
    close(ds, want.sum(0), 2.0 ** -18 * hat_of(plain).abs().sum().expand(8), "dscale")
    # Codes that were written over since cannot be differentiated.
    y = bnn.linear_q_bits(q, w)
    q.codes.zero_()
    with pytest.raises(RuntimeError):
        y.sum().backward()
    with torch.no_grad():
        assert not bnn.quantize_rows(x).codes.requires_grad and bnn.quantize_rows(x).hat is None


# ---- the block ----------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("T", ["bf16", "f32"])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M", [0, 1, 37])
def test_block(M, kind, T):
    """BinaryFeedForward on quantised rows is the chain of its calls, forwards; backwards the real block's calls at the values
    that the codes stand for."""
    T, kind = TYPES[T], KINDS[kind]
    D, F = 96, 200
    g = torch.Generator(device=DEV).manual_seed(5)
    w_in, w_out = torch.randn(2 * F, D, device=DEV, generator=g), torch.randn(D, F, device=DEV, generator=g)
    gammas = [1 + 0.2 * torch.randn(D, device=DEV, generator=g) for _ in range(3)]
    gate = (1 + 0.2 * torch.randn(1, D, device=DEV, generator=g)).to(T)
    block = bnn.BinaryFeedForward(w_in, w_out, bnn.ACT_SILU, *gammas, gate, res_scale=0.5, rows=kind)
    x = torch.randn(M, D, device=DEV, generator=g).to(T)
    n = block.first_norm(x)
    assert isinstance(n, bnn.QuantizedRows) and n.shape == (M, D)
    r, after = block.forward(x, n, keep=True)
    hat_n = bnn.dequantize_rows(n, T)
    # The same from the calls, the result of the gated product quantised apart from it.
    if kind == bnn.ROWS_MX4:
        h = bnn.gated_q_bits(n, block.w_in, block.scale_in, out_kind=kind, dtype=T)
    else:
        h = bnn.quantize_rows(bnn.gated_q_bits(n, block.w_in, block.scale_in, dtype=T), kind)
    y = bnn.linear_q_bits(h, block.w_out, block.scale_out, dtype=T)
    want_r, want_n = bnn.norm_residual_q(y, x, gate if M else None, 0.5, bnn.NORM_RMS, gammas[1], None, bnn.NORM_RMS, gammas[2], None, 1e-5, max(M, 1), kind)
    assert torch.equal(r, want_r) and torch.equal(after.codes, want_n.codes)
    dr, dn = torch.randn(M, D, device=DEV, generator=g).to(T), torch.randn(M, D, device=DEV, generator=g).to(T)
    dx, dn_before = block.backward(dr, dn)
    hat_h = bnn.dequantize_rows(h, T)
    first = bnn.norm_residual_backward(dr, dn, y, r, gate if M else None, 0.5, bnn.NORM_RMS, gammas[1], None, bnn.NORM_RMS, gammas[2], None, 1e-5, max(M, 1))
    two = bnn.linear_bits_backward(first["dy"], hat_h, block.w_out, block.scale_out)
    one = bnn.gated_bits_backward(two["dx"], hat_n, block.w_in, block.scale_in)
    assert torch.equal(dx, first["dx"]) and torch.equal(dn_before, one["dx"])
    for name, want in (("w_in", one["dw"]), ("w_out", two["dw"]), ("scale_in", one["dscale"]), ("scale_out", two["dscale"]), ("next_gamma", first["dpre_gamma"])):
        assert torch.equal(block.grads[name], want), name
    if M:
        n.codes.zero_()
        with pytest.raises(RuntimeError):
            block.backward(dr, dn)
    with pytest.raises(ValueError):
        block.forward(x, x)
    with pytest.raises(ValueError):
        bnn.BinaryFeedForward(w_in, w_out, rows=7)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_a_float32_block_of_many_values(kind):
    """600 000 hidden values, some of them next to a border between two codes: the block's are those of a float32 gated product."""
    M, D, F = 300, 256, 2000
    block = block_of(kind, D, F)
    x = torch.randn(M, D, device=DEV, generator=torch.Generator(device=DEV).manual_seed(6))
    n = block.first_norm(x)
    r, after = block.forward(x, n)
    h = bnn.gated_q_bits(n, block.w_in, block.scale_in, dtype=torch.float32, out_kind=bnn.ROWS_MX4 if kind == "mx4" else None)
    y = bnn.linear_q_bits(h if kind == "mx4" else bnn.quantize_rows(h, KINDS[kind]), block.w_out, block.scale_out, dtype=torch.float32)
    want_r, want = bnn.norm_residual_q(y, x, post=bnn.NORM_RMS, post_gamma=block.post_gamma, pre=bnn.NORM_RMS, pre_gamma=block.next_gamma, kind=KINDS[kind])
    assert torch.equal(r, want_r) and torch.equal(after.codes, want.codes)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_block_is_near_the_real_one(kind):
    """On rows that the codes hold exactly the first product is the real block's."""
    kind = KINDS[kind]
    D, F, M = 64, 96, 12
    g = torch.Generator(device=DEV).manual_seed(9)
    w_in, w_out = torch.randn(2 * F, D, device=DEV, generator=g), torch.randn(D, F, device=DEV, generator=g)
    real, coded = bnn.BinaryFeedForward(w_in, w_out), bnn.BinaryFeedForward(w_in, w_out, rows=kind)
    q = coded.first_norm(torch.randn(M, D, device=DEV, generator=g))
    n = bnn.dequantize_rows(q, torch.float32)
    a = bnn.gated_bits(n, real.w_in, real.scale_in)
    b = bnn.gated_q_bits(q, coded.w_in, coded.scale_in, dtype=torch.float32)
    size = n.abs().sum(1, keepdim=True) * real.scale_in.max()
    # |z| <= size; either z is off by (D + 12) 2^-24 size, its activation by 1.2 times that and 32 2^-24 (1 + size), h by both times size.
    assert ((a - b).abs() <= 64 * D * F32 * (1 + size) ** 2).all()


def block_of(kind, D, F):
    g = torch.Generator(device=DEV).manual_seed(21)
    return bnn.BinaryFeedForward(torch.randn(2 * F, D, device=DEV, generator=g), torch.randn(D, F, device=DEV, generator=g), rows=KINDS[kind],
                                 post_gamma=torch.rand(D, device=DEV, generator=g) + 0.5, next_gamma=torch.rand(D, device=DEV, generator=g) + 0.5)


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_a_captured_training_step(kind):
    """Forwards and backwards in one graph, replayed with new inputs and eager work between: bit for bit the eager step."""
    M, D, F = 150, 96, 200
    block = block_of(kind, D, F)
    g = torch.Generator(device=DEV).manual_seed(22)
    x, dr, dn = (torch.randn(M, D, device=DEV, generator=g).bfloat16() for _ in range(3))

    def step():
        r, after = block.forward(x, block.first_norm(x), keep=True)
        dx, dn_before = block.backward(dr, dn)
        scales = after.scales if kind == "i8" else after.scales[:, :D // 32]         # bytes past them mean nothing
        return [r, after.codes, scales, dx, dn_before, *(block.grads[k] for k in ("w_in", "w_out", "scale_in", "scale_out", "next_gamma"))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(4):
        x.copy_(torch.randn(M, D, device=DEV, generator=g).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        have = [t.clone() for t in captured]
        want = step()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(have, want)):
            assert torch.equal(a, b), i


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_two_streams_at_once(kind):
    """Calls on two streams share nothing: rows, products and norms of each come out as they do alone."""
    M, D, F = 700, 512, 1000
    block = block_of(kind, D, F)
    g = torch.Generator(device=DEV).manual_seed(23)
    xs = [torch.randn(M, D, device=DEV, generator=g).bfloat16() for _ in range(2)]
    alone = [block.forward(x, block.first_norm(x)) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(5):
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(block.forward(x, block.first_norm(x)))
    torch.cuda.synchronize()
    for i, (r, after) in enumerate(got):
        assert torch.equal(r, alone[i % 2][0]) and torch.equal(after.codes, alone[i % 2][1].codes), i
