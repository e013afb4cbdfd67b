"""The kernels behind products of quantised rows, each against the definition in 64 bits at sizes that it is taken for; and norms and
quantisation of more rows than workgroups.

FORMS names the kernel of each shape.  A host test asks the library which one it launches (nothing runs), so that a change of the rule that
chooses them cannot leave one of them without a test; the GPU tests compare the same shapes.  Rows and channels fit no tile; K ends
inside a block of 32, a step, a piece of four words and a stage of 512 elements, and takes one stage, two and many.  Tolerances are
those of test_quantised_activations.py; references are products in 64 bits on the GPU."""
import json
import re
import subprocess
import sys

import pytest
import torch

import paper_1602_02830_amd as bnn
from paper_1602_02830_amd import binding
from test_launch_limits import A, B, C, CHILD, LIB, OUT, RUNTIME, launches_of  # noqa: F401
from test_quantised_activations import INF, KINDS, MX4, NAN, check_codes, placed, result
from test_quantised_activations import test_norm as norm_against_its_definition
from test_real_activations import ACTS, DEV, F32, NORMS, ROUND, TINY, TYPES, rounded

gpu = pytest.mark.gpu

# Kernel, its tile's rows: (M, N, K).
FORMS = {
    "i8": {
        ("waves", 32): [(6000, 258, 257), (300, 4094, 333), (1000, 1030, 400), (1000, 520, 785), (1500, 258, 1025), (200, 1538, 1300), (1500, 130, 4128)],
        ("tile", 64): [(1000, 8190, 352), (3500, 2050, 417), (3500, 2050, 449), (1000, 4094, 545), (1000, 4094, 580), (450, 8190, 640), (2050, 1538, 785),
                       (5100, 520, 1024), (5100, 520, 1025), (5100, 520, 1057), (5100, 520, 1100), (257, 8190, 1569), (1000, 2050, 2085), (6000, 258, 3333)],
        ("tile", 128): [(5100, 3070, 320), (5100, 3070, 333), (3500, 4094, 384), (6000, 2050, 417), (5100, 2050, 545), (5100, 2050, 580), (8200, 1030, 785),
                        (6000, 2050, 1024), (6000, 2050, 1025), (6000, 2050, 1057), (6000, 2050, 1100), (6000, 520, 2085), (6000, 520, 3333)],
    },
    "mx4": {
        ("waves", 32): [(4100, 4094, 290), (3500, 2050, 333), (1500, 2050, 417), (450, 4094, 545), (1000, 1030, 785), (2600, 258, 1025), (200, 3070, 1153),
                        (3500, 130, 2085), (2600, 130, 3333)],
        ("waves", 64): [(6000, 130, 2500), (1000, 1030, 3333), (513, 2050, 4128)],
        ("tile", 64): [(1000, 8190, 400), (1000, 8190, 417), (2600, 3070, 449), (3500, 2050, 545), (3500, 2050, 640), (450, 8190, 785), (450, 8190, 1024),
                       (450, 8190, 1025), (513, 6150, 1057), (2050, 1538, 1100), (3000, 1030, 1153), (300, 8190, 2085), (1000, 2050, 3333)],
        ("tile", 128): [(5100, 3070, 290), (5100, 3070, 333), (3500, 4094, 352), (3500, 4094, 384), (3500, 4094, 417), (3000, 4094, 545), (3000, 4094, 640),
                        (5100, 2050, 785), (6000, 2050, 1024), (6000, 2050, 1025), (6000, 2050, 1057), (6000, 2050, 1100), (6000, 2050, 2085),
                        (3500, 1030, 3333)],
    },
}
ALL = [(kind, form, *size) for kind, forms in FORMS.items() for form, sizes in forms.items() for size in sizes]


# ---- which kernel a call takes ---------------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def kernels_of(tmp_path_factory):
    """calls -> the name of each call's one kernel as the library has it; calls that are refused or launch more fail."""
    folder = tmp_path_factory.mktemp("kernels")
    line = "launch_log[launches][2] = *(uint64_t*)args[0];"
    assert line in RUNTIME
    src, so = folder / "runtime.c", folder / "runtime.so"
    src.write_text("#define _GNU_SOURCE\n#include <dlfcn.h>\n#include <stdio.h>\n" +
                   RUNTIME.replace(line, 'Dl_info at; fprintf(stderr, "kernel %s\\n", dladdr(f, &at) && at.dli_sname ? at.dli_sname : "?");'))
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", str(src), "-o", str(so), "-ldl"], check=True)

    def run(*calls):
        r = subprocess.run([sys.executable, "-c", CHILD, str(so), LIB], input=json.dumps([[n, list(a)] for n, a in calls]),
                           stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
        assert r.returncode == 0, r.stderr
        assert all(st == 0 and len(log) == 1 for st, log in json.loads(r.stdout))
        names = [s[7:] for s in r.stderr.splitlines() if s.startswith("kernel ")]
        assert len(names) == len(calls)
        return names

    return run


def library_call(kind, gated, M, N, K, type_, coded=False):
    """A call with the leading dimensions of rows that lie one behind another."""
    blocks, F = (K + 31) // 32, N // 2
    rows = KINDS[kind]
    x = (rows, A, blocks * (32 if kind == "i8" else 16), B, (blocks + 15) // 16 * 16, C, blocks, 0, 0, 0, type_)
    if not gated:
        return "bnn_linear_q_bits", (*x, 0, 0, OUT, N, M, N, K, 0)
    out = (OUT + (1 << 43), (F + 31) // 32 * 16, OUT + (3 << 42), (F + 511) // 512 * 16) if coded else (0, 0, 0, 0)
    return "bnn_gated_q_bits", (*x, OUT, F, *out, M, F, K, 0)


def form_of(name):
    """(kind, gated, (kernel, rows of its tile)) of a kernel's name."""
    m = re.fullmatch(r"_ZN3bnn\d+q_(waves|tile)_kernelILi(\d)ELi(\d)ELi(\d)EEEvNS_12QProductArgsE", name)
    assert m, name
    return ("i8", "mx4")[int(m[2])], m[3] == "1", (m[1], 32 * int(m[4]))


@pytest.mark.parametrize("kind,form,M,N,K", ALL)
def test_shapes_take_the_kernel_that_they_are_here_for(kernels_of, kind, form, M, N, K):
    """Whatever the result's type, and whether it is gated, real or quantised."""
    assert N % 2 == 0
    calls = [(gated, library_call(kind, gated, M, N, K, type_, coded)) for type_ in range(3) for gated, coded in ((False, False), (True, False), (True, True))]
    for (gated, _), name in zip(calls, kernels_of(*(c for _, c in calls))):
        assert form_of(name) == (kind, gated, form)


# ---- against the definition -------------------------------------------------------------------------------------------

class Product:
    """Operands and definition of a product, made on the GPU; `far` are the same rows further apart, with junk between them and in the bytes
    of scales that mean nothing.  Weights have junk in pad bits and pad words.  of(): which of scale and bias a call has."""

    def __init__(self, M, N, K, kind):
        self.kind = KINDS[kind]
        g = torch.Generator(device=DEV).manual_seed(M + 7 * N + 31 * K)
        x = torch.randn(M, K, device=DEV, generator=g) * (1 + 15 * (torch.rand(K, device=DEV, generator=g) < 0.02).float())
        x[M // 2] *= 2.0 ** -9
        self.q = bnn.quantize_rows(x, self.kind)
        blocks, c, s = (K + 31) // 32, self.q.codes, self.q.scales
        codes = torch.full((M, c.shape[1] + 16), 0xFF, dtype=torch.uint8, device=DEV)
        codes[:, :c.shape[1]] = c
        if kind == "mx4":
            scales = torch.full((M, s.shape[1] + 16), 0xFF, dtype=torch.uint8, device=DEV)
            scales[:, :blocks] = s[:, :blocks]
            s = scales[:, :s.shape[1]]
        self.far = bnn.QuantizedRows(self.kind, K, codes[:, :c.shape[1]], s)
        codes, steps = decoded(self.q)
        self.x = (codes * steps[:, :, None]).reshape(M, 32 * blocks)[:, :K]
        bits = torch.randint(0, 2, (N, 32 * blocks), device=DEV, generator=g)
        self.w = 2.0 * bits[:, :K].double() - 1
        bits[:, K:] = 1
        words = (bits.view(N, blocks, 32) << torch.arange(32, device=DEV)).sum(2)
        self.wd = torch.full((N, blocks + 3), 0x5A5A5A5A, dtype=torch.int32, device=DEV)[:, :blocks]
        self.wd.copy_(torch.where(words >= 1 << 31, words - (1 << 32), words))
        self.sums, self.size = self.x @ self.w.t(), self.x.abs().sum(1, keepdim=True)
        self.some = (torch.rand(N, device=DEV, generator=g) + 0.5) / K ** 0.5, 0.3 * torch.randn(N, device=DEV, generator=g)

    def of(self, scale, bias):
        self.scale, self.bias = self.some[0] if scale else None, self.some[1] if bias else None
        return self.scale, self.bias

    def z(self):
        """z and a bound of its error."""
        a = self.scale.double() if self.scale is not None else 1.0
        z = self.sums * a + (self.bias.double() if self.bias is not None else 0.0)
        # 8 bits: the sum is exact; to float, times the row's scale, times the channel's and bias in one.
        es = 2 * F32 * self.sums.abs() if self.kind == bnn.ROWS_I8 else (self.x.shape[1] + 8) * F32 * self.size
        return z, 1.01 * es * a + F32 * (z.abs() + es * a)


def near(got, want, tol, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:5].tolist())


def decoded(q):
    """Codes [M][blocks][32] and scales [M][blocks] of quantised rows, in float64 on the GPU."""
    M, blocks = q.shape[0], (q.K + 31) // 32
    if q.kind == bnn.ROWS_I8:
        c = q.codes[:, :32 * blocks].view(torch.int8).reshape(M, blocks, 8, 4).transpose(2, 3)           # byte 4 i + j: element 8 j + i
        return c.reshape(M, blocks, 32).double(), q.scales.double()[:, None].expand(M, blocks)
    raw = q.codes[:, :16 * blocks]
    nibbles = torch.stack([raw & 15, raw >> 4], dim=-1).view(M, blocks, 4, 8).transpose(2, 3).reshape(M, blocks, 32)      # nibble 8 i + j: element 4 j + i
    c = MX4.to(DEV)[(nibbles & 7).long()] * torch.where(nibbles > 7, -1.0, 1.0).double()
    s = q.scales[:, :blocks].double()
    return c, torch.where(s == 255, torch.full_like(s, NAN), torch.exp2(s - 127))


def quantised_near(q, v, err, what):
    """4-bit rows of values that are known but for err: the scale such that the largest magnitude fits, the codes as near as any, the
    block's rest zero.  (As test_quantised_activations.nearest_but_for.)"""
    c, s = decoded(q)
    pad = (0, 32 * c.shape[1] - q.K)
    v, err = (torch.nn.functional.pad(t, pad).view(c.shape) for t in (v, err))
    most, e = v.abs().amax(2), err.amax(2)
    assert ((most - e < 7 * s) & ((most + e >= 3.5 * s) | (s == 2.0 ** -126))).all(), (what, "scales")
    best = torch.full_like(v, INF)
    for code in MX4.tolist():
        best = torch.minimum(best, (v.abs() - code * s[:, :, None]).abs())
    # 2^-20 of a step: what the comparison itself rounds.
    bad = ~((c * s[:, :, None] - v).abs() <= best + 2 * err + 2.0 ** -20 * s[:, :, None])
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:5].tolist())
    if pad[1]:
        assert (c[:, -1, 32 - pad[1]:] == 0).all(), (what, "pad")


@gpu
@pytest.mark.parametrize("kind,form,M,N,K", ALL)
def test_linear_of_each_form(kind, form, M, N, K):
    p = Product(M, N, K, kind)
    for T, act, scale, bias, res in ((torch.bfloat16, "none", True, True, True), (torch.float32, "gelu", True, False, False), (torch.float16, "silu", True, True, False),
                                     (torch.float32, "none", False, False, True)):
        vectors = p.of(scale, bias)
        x = p.far if T == torch.float16 else p.q
        r = torch.randn(M, N, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(T) if res else None
        want, err = result(p, act, residual=r)
        y = bnn.linear_q_bits(x, p.wd, *vectors, ACTS[act], placed(r, 3, 1) if res else None, T)
        near(y, want, rounded(want, err, T), (T, act))
        if res:                                                 # in the residual's place, and between the columns of a wider result
            place = r.clone()
            assert bnn.linear_q_bits(x, p.wd, *vectors, ACTS[act], place, out=place) is place
            assert torch.equal(place, y)
            wide = torch.full((M + 2, N + 5), 7.0, dtype=T, device=DEV)
            bnn.linear_q_bits(x, p.wd, *vectors, ACTS[act], r, out=wide[1:-1, 3:-2])
            assert torch.equal(wide[1:-1, 3:-2], y)
            assert (wide[0] == 7).all() and (wide[-1] == 7).all() and (wide[:, :3] == 7).all() and (wide[:, -2:] == 7).all()


@gpu
@pytest.mark.parametrize("kind,form,M,N,K", ALL)
def test_gated_of_each_form(kind, form, M, N, K):
    F, p = N // 2, Product(M, N, K, kind)
    for T, act, scale, bias in ((torch.bfloat16, "silu", True, False), (torch.float32, "gelu_tanh", True, True), (torch.float16, "sigmoid", True, True)):
        vectors = p.of(scale, bias)
        x = p.far if T == torch.float16 else p.q
        want, err = result(p, act, gated=True)
        near(bnn.gated_q_bits(x, p.wd, *vectors, ACTS[act], T), want, rounded(want, err, T), (T, act))
        # Quantised for the product that follows, with and without h^, nothing written behind a row's codes.
        q = bnn.gated_q_bits(x, p.wd, *vectors, ACTS[act], T, out_kind=bnn.ROWS_MX4, hat=True)
        quantised_near(q, want, err, (T, act, "h^"))
        assert torch.equal(q.hat, bnn.dequantize_rows(q, T))
        blocks = (F + 31) // 32
        codes = torch.full((M + 1, 16 * blocks + 32), 0xA5, dtype=torch.uint8, device=DEV)
        scales = torch.full((M + 1, (blocks + 15) // 16 * 16), 0xA5, dtype=torch.uint8, device=DEV)
        only = bnn.QuantizedRows(bnn.ROWS_MX4, F, codes[:M, :16 * blocks], scales[:M])
        assert bnn.gated_q_bits(x, p.wd, *vectors, ACTS[act], T, out_q=only) is only
        assert torch.equal(only.codes, q.codes[:, :16 * blocks]) and torch.equal(only.scales[:, :blocks], q.scales[:, :blocks])
        assert (codes[M] == 0xA5).all() and (codes[:, 16 * blocks:] == 0xA5).all() and (scales[M] == 0xA5).all() and (scales[:, blocks:] == 0xA5).all()


def exact_sums(M, N, K, kind):
    """Rows whose sums float32 holds exactly in any order: every element and every sign counts, to the last bit.  8 bits: whole numbers
    up to 127 with scales that are powers of two; 4 bits: codes with four scales, multiples of 1/2 below 48 K < 2^19."""
    p = Product(M, N, K, kind)
    g = torch.Generator(device=DEV).manual_seed(2)
    if kind == "i8":
        x = torch.randint(-126, 127, (M, K), device=DEV, generator=g).double()
        x[torch.arange(M, device=DEV), torch.randint(0, K, (M,), device=DEV, generator=g)] = 127
        x *= torch.exp2(torch.randint(-4, 5, (M, 1), device=DEV, generator=g).double())
    else:
        x = MX4.to(DEV)[torch.randint(0, 8, (M, K), device=DEV, generator=g)] * (2.0 * torch.randint(0, 2, (M, K), device=DEV, generator=g) - 1)
        x[:, ::32] = 6                       # a block's largest magnitude, from which its scale is
        x *= torch.exp2(torch.randint(0, 4, (M, (K + 31) // 32), device=DEV, generator=g).double()).repeat_interleave(32, 1)[:, :K]
    q = bnn.quantize_rows(x.float(), KINDS[kind])
    c, steps = decoded(q)
    assert torch.equal((c * steps[:, :, None]).reshape(M, -1)[:, :K], x)
    sums = x @ p.w.t()
    assert torch.equal(bnn.linear_q_bits(q, p.wd, dtype=torch.float32).double(), sums)
    if N % 2 == 0:
        h = sums[:, :N // 2] * sums[:, N // 2:]
        assert torch.equal(bnn.gated_q_bits(q, p.wd, act=ACTS["none"], dtype=torch.float32), h.float())


@gpu
@pytest.mark.parametrize("kind,form,M,N,K", ALL)
def test_exact_sums_of_each_form(kind, form, M, N, K):
    exact_sums(M, N, K, kind)


#: Tiles of 16 rows: runs of 512 elements by one wavefront to eight and more, that end inside a block of 32 and a piece of four.
SMALL = [(1, 64, 32), (3, 18, 40), (16, 48, 512), (2, 34, 513), (5, 100, 1030), (17, 96, 4096), (8, 40, 8200), (33, 130, 700), (1, 8192, 4096), (9, 20, 5000),
         (16, 200, 1057), (40, 64, 1569), (66, 33, 545), (80, 1800, 97), (100, 1002, 333), (1, 2, 1)]


@pytest.mark.parametrize("kind", list(KINDS))
def test_few_rows_take_small_tiles(kernels_of, kind):
    names = kernels_of(*(library_call(kind, gated, M, N, K, 0) for M, N, K in SMALL for gated in (False, True) if not gated or N % 2 == 0))
    assert all("q_small_kernel" in name for name in names)
    assert len(set(names)) == 4              # one block of channels and two, linear and gated


@gpu
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,N,K", SMALL)
def test_exact_sums_of_small_tiles(M, N, K, kind):
    exact_sums(M, N, K, kind)


@gpu
@pytest.mark.parametrize("kind,form,M,N,K", [(kind, form, *sizes[-1]) for kind, forms in FORMS.items() for form, sizes in forms.items()])
def test_nan_rows_of_each_form(kind, form, M, N, K):
    """A row (8 bits) or block (4 bits) that stands for NaN makes its own row of the result NaN, and no other."""
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(M, K, device=DEV, generator=g)
    bad = [3, 40, M // 2, M - 1]
    x[3, 77], x[40, 0], x[M // 2, K // 2], x[M - 1, K - 1] = NAN, INF, -INF, NAN
    w = bnn.pack_sign(torch.randn(N, K, device=DEV, generator=g))
    q = bnn.quantize_rows(x, KINDS[kind])
    y = bnn.linear_q_bits(q, w)
    there = torch.isnan(y)
    assert there.any(1).nonzero().flatten().tolist() == bad and there.all(1).nonzero().flatten().tolist() == bad
    h = bnn.gated_q_bits(q, w, out_kind=bnn.ROWS_MX4, hat=True)
    assert torch.isnan(h.hat).any(1).nonzero().flatten().tolist() == bad and torch.isnan(h.hat).all(1).nonzero().flatten().tolist() == bad


# ---- rows that are walked over ------------------------------------------------------------------------------------------
# Workgroups of the norms and of the quantisation to 8 bits take one row after another; from the third on they use every buffer again.

#: (M, D) of rows in 1, 1, 1, 3, 4, 5, 8, 16 and 16 wavefronts: three rows a workgroup and more.
WALKED = [(13000, 5), (13000, 300), (13000, 777), (4200, 2049), (3300, 4096), (2600, 5000), (1700, 8192), (600, 9001), (600, 16384)]
#: And of rows that are read twice.
LONG = (1100, 16385)
PART = 200                                   # rows of which no workgroup has a second one


def quantise_call(kind, type_, M, K):
    blocks = (K + 31) // 32
    return "bnn_quantize_rows", (KINDS[kind], type_, A, K, B, blocks * 32, C, (blocks + 15) // 16 * 16, 0, 0, M, K, 0)


def norm_call(kind, type_, M, D, beta):
    """Without its two floats, which travel in registers of their own."""
    blocks = (D + 31) // 32
    return "bnn_norm_residual_q", (type_, A, D, 0, 0, 0, 0, 1, 2, 0, beta, 2, 0, beta, 0, 0, KINDS[kind], B, blocks * 32, C, (blocks + 15) // 16 * 16, 0, 0, M, D, 0)


def test_workgroups_take_rows_one_after_another(launches_of):  # noqa: F811
    for type_ in range(3):
        for M, D in [*WALKED, LONG]:
            calls = [quantise_call("i8", type_, M, D)]
            if (M, D) != LONG:
                calls += [norm_call(kind, type_, M, D, beta) for kind in KINDS for beta in (0, OUT)]
            for (st, log), (name, _) in zip(launches_of(*calls), calls):
                assert st == 0 and len(log) == 1 and PART <= log[0][0] and 2 * log[0][0] < M, (name, M, D, log)


def part_of(q, a, b):
    return bnn.QuantizedRows(q.kind, q.K, q.codes[a:b], q.scales[a:b], None if q.hat is None else q.hat[a:b])


def same_rows(q, own, what):
    blocks = (q.K + 31) // 32
    assert torch.equal(q.codes, own.codes) and torch.equal(q.hat, own.hat), what
    assert torch.equal(q.scales, own.scales) if q.kind == bnn.ROWS_I8 else torch.equal(q.scales[:, :blocks], own.scales[:, :blocks]), what


def rows_of_many_sizes(M, D, T, seed):
    """Rows whose magnitudes differ: what is left of another row shows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(M, D, device=DEV, generator=g) * torch.exp2(torch.randint(-6, 7, (M, 1), device=DEV, generator=g).float())
    x[5 % M] = 0
    return x.to(T)


@gpu
@pytest.mark.parametrize("T", list(TYPES))
@pytest.mark.parametrize("M,D", [*WALKED, LONG])
def test_quantise_more_rows_than_workgroups(M, D, T):
    """Each row is what it is by itself, bit for bit; the first, some and the last against the definition, with x^ in the rows' own
    place too."""
    x = rows_of_many_sizes(M, D, TYPES[T], 1)
    q = bnn.quantize_rows(x, bnn.ROWS_I8, hat=True)
    for a in range(0, M, PART):
        same_rows(part_of(q, a, a + PART), bnn.quantize_rows(x[a:a + PART], bnn.ROWS_I8, hat=True), a)
    for a in (0, M // 2 + 3, M - 16):
        check_codes(part_of(q, a, a + 16), x[a:a + 16].cpu())
    place = bnn.QuantizedRows(bnn.ROWS_I8, D, torch.empty_like(q.codes), torch.empty_like(q.scales), x)
    same_rows(bnn.quantize_rows(x, out=place), q, "in place")


@gpu
@pytest.mark.parametrize("T,post,pre,gate_rows", [("bf16", "layer", "rms", 7), ("f16", "rms", "layer", 2500), ("f32", "rms", "rms", 0), ("f32", "layer", "layer", 1)])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("M,D", WALKED)
def test_norms_of_more_rows_than_workgroups(M, D, kind, T, post, pre, gate_rows):
    """r, codes, scales and n^ of each row are what it gets by itself, bit for bit, with a gate whose row changes on the way; with r in the
    stream's place too.  Gammas and betas begin at any multiple of four bytes."""
    T, kind = TYPES[T], KINDS[kind]
    y, x = rows_of_many_sizes(M, D, T, 2), rows_of_many_sizes(M, D, T, 3)
    g = torch.Generator(device=DEV).manual_seed(4)
    R = gate_rows or M
    gate = (1 + 0.3 * torch.randn(-(-M // R), D, device=DEV, generator=g)).to(T) if gate_rows else None
    per_row = gate.repeat_interleave(R, 0)[:M] if gate_rows else None
    vectors = [torch.randn(D + 1, device=DEV, generator=g)[i % 2:D + i % 2] for i in range(4)]
    post_args = (NORMS[post], vectors[0], vectors[1] if post == "layer" else None)
    pre_args = (NORMS[pre], vectors[2], vectors[3] if pre == "layer" else None, 1e-5)
    r, q = bnn.norm_residual_q(y, x, gate, 0.5, *post_args, *pre_args, R, kind, hat=True)
    real_r, n = bnn.norm_residual(y, x, gate, 0.5, *post_args, *pre_args, R)
    assert torch.equal(r, real_r)
    for a in range(0, M, PART):
        b = min(a + PART, M)
        own_r, own = bnn.norm_residual_q(y[a:b], x[a:b], per_row[a:b] if gate_rows else None, 0.5, *post_args, *pre_args, 1, kind, hat=True)
        assert torch.equal(own_r, r[a:b]), a
        same_rows(part_of(q, a, b), own, a)
    place = x.clone()
    got = bnn.norm_residual_q(y, place, gate, 0.5, *post_args, *pre_args, R, out=place, out_q=bnn.quantized_rows(M, D, kind, DEV, T))
    assert torch.equal(place, r)
    same_rows(got[1], q, "in place")
    # Codes are those of n but for its rounding: half a step, and half a unit of n and of n^ (two norms are equal to 2^-20 of the row).
    c, s = decoded(q)
    value = (c * s[:, :, None]).reshape(M, -1)[:, :D]
    step = (s if kind == bnn.ROWS_I8 else 2 * s)[:, :, None].expand(c.shape).reshape(M, -1)[:, :D]
    n = n.double()
    assert ((value - n).abs() <= 0.5 * step + ROUND[T] * n.abs() + 2.0 ** -20 * n.abs().amax(1, keepdim=True) + TINY[T]).all()


@gpu
@pytest.mark.parametrize("T", list(TYPES))
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("post,pre", [("layer", "layer"), ("none", "layer"), ("layer", "none")])
def test_norms_of_long_rows_with_betas(post, pre, kind, T):
    """Past 8192 elements, against the definition."""
    norm_against_its_definition(3, 9001, post, pre, True, kind, T)


# ---- matrices past 2^31 elements ------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_matrices_of_more_than_2_31_elements(kind):
    """Rows, results, codes and x^ on both sides of the 2^31st element, and the last ones, are what they are in a small call.  Sums are exact."""
    M, K, N, kind = (1 << 19) + 700, 4128, 4160, KINDS[kind]
    assert M * K > 1 << 31 < M * N
    g = torch.Generator(device=DEV).manual_seed(8)
    few = torch.randint(-6, 7, (1000, K), device=DEV, generator=g).bfloat16()
    few[:, ::32] = 6 if kind == bnn.ROWS_MX4 else 127             # steps of 1
    few[few.abs() == 5] = 4                                       # not a code of 4 bits
    x = few[torch.arange(M, device=DEV) % 1000]
    w, gate = bnn.pack_sign(torch.randn(N, K, device=DEV, generator=g)), bnn.pack_sign(torch.randn(2 * N, K, device=DEV, generator=g))
    q = bnn.quantize_rows(x, kind, hat=True)
    assert torch.equal(q.hat, x) and torch.equal(bnn.dequantize_rows(q, torch.bfloat16), x)
    r, n = bnn.norm_residual_q(x, x, None, 0.5, pre=bnn.NORM_RMS, kind=kind, hat=True)
    y = bnn.linear_q_bits(q, w, dtype=torch.float32)
    h = bnn.gated_q_bits(q, gate, act=ACTS["none"], dtype=torch.bfloat16)
    hq = bnn.gated_q_bits(q, gate, act=ACTS["none"], dtype=torch.bfloat16, out_kind=bnn.ROWS_MX4, hat=True)
    assert torch.equal(bnn.dequantize_rows(hq, torch.bfloat16), hq.hat)
    for a in (0, (1 << 31) // N - 100, (1 << 31) // K - 100, M - 200):
        b = a + 200
        own = bnn.quantize_rows(x[a:b], kind, hat=True)
        same_rows(part_of(q, a, b), own, a)
        own_r, own_n = bnn.norm_residual_q(x[a:b], x[a:b], None, 0.5, pre=bnn.NORM_RMS, kind=kind, hat=True)
        assert torch.equal(r[a:b], own_r), a
        same_rows(part_of(n, a, b), own_n, a)
        assert torch.equal(y[a:b], bnn.linear_q_bits(own, w, dtype=torch.float32)), a
        assert torch.equal(h[a:b], bnn.gated_q_bits(own, gate, act=ACTS["none"], dtype=torch.bfloat16)), a
        same_rows(part_of(hq, a, b), bnn.gated_q_bits(own, gate, act=ACTS["none"], dtype=torch.bfloat16, out_kind=bnn.ROWS_MX4, hat=True), a)


@gpu
def test_more_groups_than_one_launch_of_4_bit_rows_holds():
    """2^31 groups of eight elements and more: rows of one element, quantised and made reals of again."""
    M = (1 << 29) + 1000
    x = torch.randint(-4, 5, (M, 1), device=DEV, dtype=torch.int8, generator=torch.Generator(device=DEV).manual_seed(9)).bfloat16()
    q = bnn.quantize_rows(x, bnn.ROWS_MX4, hat=True)              # every number up to 4 is a code times a power of two
    assert torch.equal(q.hat, x)
    assert torch.equal(bnn.dequantize_rows(q, torch.bfloat16), x)


# ---- nothing ----------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("kind", [*KINDS, "real"])
@pytest.mark.parametrize("M,N,K", [(0, 64, 96), (5, 0, 96), (5, 64, 0)])
def test_gradients_of_nothing(M, N, K, kind, native, monkeypatch):
    """No rows, no channels, no elements: gradients of the inputs' sizes, of zeros where nothing comes in; of real rows too."""
    if not native:
        monkeypatch.setattr(binding, "_calls", None)
    x = torch.randn(M, K, device=DEV, requires_grad=True)
    w = torch.zeros(N, (K + 31) // 32, dtype=torch.int32, device=DEV)
    s, b = (torch.ones(N, device=DEV, requires_grad=True) for _ in range(2))
    if kind == "real":
        results = [bnn.linear_bits(x, w, s, b), bnn.gated_bits(x, w, s, b, ACTS["none"])]
    else:
        q = bnn.quantize_rows(x, KINDS[kind])
        results = [bnn.linear_q_bits(q, w, s, b), bnn.gated_q_bits(q, w, s, b, ACTS["none"]),
                   bnn.gated_q_bits(q, w, s, b, ACTS["none"], out_kind=bnn.ROWS_MX4).hat]
    for y in results:
        dx, ds, db = torch.autograd.grad(y, (x, s, b), torch.ones_like(y), retain_graph=True)
        assert dx.shape == x.shape and ds.shape == s.shape and db.shape == b.shape
        assert (dx == 0).all() and (K > 0 or (ds == 0).all())


@gpu
@pytest.mark.parametrize("native", [True, False])
def test_norm_gradients_of_rows_of_nothing(native, monkeypatch):
    if not native:
        monkeypatch.setattr(binding, "_calls", None)
    y, gamma, beta = (torch.randn(*s, device=DEV, requires_grad=True) for s in ((5, 0), (0,), (0,)))
    for n in (bnn.norm_residual(y, pre=bnn.NORM_LAYER, pre_gamma=gamma, pre_beta=beta)[1],
              bnn.norm_residual_q(y, pre=bnn.NORM_LAYER, pre_gamma=gamma, pre_beta=beta)[1].hat):
        assert [g.shape for g in torch.autograd.grad(n, (y, gamma, beta), torch.ones_like(n))] == [(5, 0), (0,), (0,)]
