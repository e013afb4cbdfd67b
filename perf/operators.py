"""The feed-forward block of a language model with one-bit weights: three operators, each with its backward pass.

Activations are real (bfloat16, float16 or float32), weights are the package's packed +-1 rows with a real scale per
output channel (``s_n = scale_n * sum_k x_k w_nk``).

  linear   y = act(scale * (x w^T) + bias) + residual                       bnn.linear_bits
  gated    h = act(z_gate) * z_up, z = scale * (x w^T) + bias, w [2F][K]     bnn.gated_bits
  norm     r = x + res_scale * gate * post(y),  n = pre(r)                   bnn.norm_residual

post and pre are a root-mean-square norm, a layer norm or nothing.  A case with ``"back": True`` is the backward pass: from
the gradients of the results to those of every input (of the +-1 weights as if they were real numbers, which is what
a straight-through estimator wants).

``own`` says which form run() computes: elementary torch operations in 32 bits, or the package's entry points.  The
weights are the same +-1 matrix for both; each form keeps them the way a program that calls it would (float32 for the plain
form, so that it is not charged with unpacking; packed bits for the package).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}

MAX_FLOPS = 6 * 4096 * 4096 * 16384        # the largest listed product work (gated_back_4096x4096x8192)
MAX_REALS = 16384 * 4096                   # elements of the largest listed matrix of the norms
MAX_PRODUCT_REALS = 16384 * 8192           # elements of the largest matrix of a drawn product
OTHERS = 3072                              # rows of colour images: the first layer on bytes has them (cases.py), not these


def listed():
    return [
        # One token through the block of a served model: the time of one call counts.
        {"name": "gated_1x4096x8192_bf16", "op": "gated", "back": False, "type": "bf16", "M": 1, "K": 4096, "F": 8192,
         "act": "silu", "scale": True, "bias": False},
        # A ragged prompt with sizes that fit no tile: K no multiple of 32, F odd, rows of odd length.
        {"name": "gated_333x1000x2047_f16", "op": "gated", "back": False, "type": "f16", "M": 333, "K": 1000, "F": 2047,
         "act": "gelu_tanh", "scale": True, "bias": True},
        # Long prompts, or the forward half of a training step.
        {"name": "gated_8192x4096x8192_bf16", "op": "gated", "back": False, "type": "bf16", "M": 8192, "K": 4096, "F": 8192,
         "act": "silu", "scale": True, "bias": False},
        # A small training step with odd sizes.
        {"name": "gated_back_500x784x1531_f16", "op": "gated", "back": True, "type": "f16", "M": 500, "K": 784, "F": 1531,
         "act": "gelu", "scale": True, "bias": True},
        # The backward half of a training step.
        {"name": "gated_back_4096x4096x8192_bf16", "op": "gated", "back": True, "type": "bf16", "M": 4096, "K": 4096, "F": 8192,
         "act": "silu", "scale": True, "bias": False},
        # The block's second product for a few sequences, a token each, added to the stream.
        {"name": "linear_8x8192x4096_bf16", "op": "linear", "back": False, "type": "bf16", "M": 8, "K": 8192, "N": 4096,
         "act": "none", "scale": True, "bias": True, "residual": True},
        # A layer of the framework's MLP on real inputs as they are (not binarized), in its own 32 bits.
        {"name": "linear_1000x784x4096_f32", "op": "linear", "back": False, "type": "f32", "M": 1000, "K": 784, "N": 4096,
         "act": "relu", "scale": True, "bias": True, "residual": False},
        # The block's second product for long prompts.
        {"name": "linear_8192x8192x4096_bf16", "op": "linear", "back": False, "type": "bf16", "M": 8192, "K": 8192, "N": 4096,
         "act": "none", "scale": True, "bias": False, "residual": True},
        # Its backward pass in a training step.
        {"name": "linear_back_4096x8192x4096_bf16", "op": "linear", "back": True, "type": "bf16", "M": 4096, "K": 8192, "N": 4096,
         "act": "none", "scale": True, "bias": True},
        # Between two blocks, a token at a time.
        {"name": "norm_1x4096_f16", "op": "norm", "back": False, "type": "f16", "M": 1, "D": 4096, "rows_per_gate": 1,
         "x": True, "gate": True, "post": "rms", "pre": "rms"},
        # Between two blocks of a long batch, one gate for all rows.
        {"name": "norm_16384x4096_bf16", "op": "norm", "back": False, "type": "bf16", "M": 16384, "D": 4096,
         "rows_per_gate": 16384, "x": True, "gate": True, "post": "rms", "pre": "rms"},
        # The same step backwards, in 32 bits, with layer norms, a gate for each 100 rows and rows of odd length.
        {"name": "norm_back_10000x2049_f32", "op": "norm", "back": True, "type": "f32", "M": 10000, "D": 2049,
         "rows_per_gate": 100, "x": True, "gate": True, "post": "layer", "pre": "layer"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, step):
    """A size in [lo, hi], spread over its logarithm; half of the time a multiple of `step`."""
    v = _log_int(rng, lo, hi)
    return max(step, v // step * step) if rng.random() < 0.5 else v


def draw(rng):
    while True:
        op = rng.choice(["linear", "gated", "norm"])
        kind = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
        back = rng.random() < 0.4
        if op == "norm":
            M = _log_int(rng, 1, 32768)
            case = {"op": op, "back": back, "type": kind, "M": M, "D": _size(rng, 64, 8192, 64),
                    "rows_per_gate": rng.choice([1, M, _log_int(rng, 1, M)]), "x": rng.random() < 0.8,
                    "gate": rng.random() < 0.6, "post": rng.choice(["none", "rms", "layer"]), "pre": rng.choice(["none", "rms", "layer"])}
            if case["M"] * case["D"] <= MAX_REALS and OTHERS not in case.values():
                return case
            continue
        M = _log_int(rng, 1, 16) if not back and rng.random() < 0.25 else _log_int(rng, 16, 16384)
        # The gradient of relu jumps at 0, and on which side of it a sum falls is a matter of rounding: only forward.
        acts = ["silu", "gelu", "gelu_tanh", "sigmoid"] + ([] if back else ["relu"])
        case = {"op": op, "back": back, "type": kind, "M": M, "K": _size(rng, 256, 8192, 128)}
        if op == "gated":
            case.update(F=_size(rng, 256, 8192, 128), act=rng.choice(acts), scale=True, bias=rng.random() < 0.4)
            n = 2 * case["F"]
        else:
            n = _size(rng, 256, 8192, 128)
            case.update(N=n, act=rng.choice(["none", "none"] + acts), scale=rng.random() < 0.8, bias=rng.random() < 0.5)
            if not case["scale"] and case["act"] != "none":
                case["scale"] = True
            if not back:
                case["residual"] = rng.random() < 0.5
        if work(case)["flops"] <= MAX_FLOPS and M * max(n, case["K"]) <= MAX_PRODUCT_REALS and OTHERS not in case.values():
            return case


# ---- inputs ------------------------------------------------------------------------------------------------

def _draws(case, seed):
    """The values behind a case, in the types in which a program holds them; +-1 weights as float32."""
    g = torch.Generator(device=DEV).manual_seed(1000003 * int(seed) + 7)
    T = TYPES[case["type"]]
    M = case["M"]

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=DEV).mul_(std).add_(mean).to(dtype)

    d = {}
    if case["op"] == "norm":
        D = case["D"]
        loud = 1 + 15 * (torch.rand(D, generator=g, device=DEV) < 0.01).float()      # a few channels are much larger
        d["y"] = (normal(M, D) * loud).to(T)
        d["x"] = normal(M, D, std=2.0, dtype=T) if case["x"] else None
        d["gate"] = normal(-(-M // case["rows_per_gate"]), D, std=0.3, mean=1.0, dtype=T) if case["gate"] else None
        d["res_scale"] = 0.5
        for side in ("post", "pre"):
            d[side + "_gamma"] = normal(D, std=0.2, mean=1.0) if case[side] != "none" else None
            d[side + "_beta"] = normal(D, std=0.2) if case[side] == "layer" else None
        if case["back"]:
            d["dr"] = normal(M, D, std=0.05, dtype=T)
            d["dn"] = normal(M, D, std=0.05, dtype=T) if case["pre"] != "none" else None
        return d
    K, N = case["K"], 2 * case["F"] if case["op"] == "gated" else case["N"]
    d["x"] = normal(M, K, dtype=T)
    d["w"] = torch.randint(0, 2, (N, K), generator=g, device=DEV).mul_(2).sub_(1).float()
    d["scale"] = torch.rand(N, generator=g, device=DEV).add_(0.5).div_(math.sqrt(K)) if case["scale"] else None
    d["bias"] = normal(N, std=0.2) if case["bias"] else None
    if case["back"]:
        d["dy"] = normal(M, case["F"] if case["op"] == "gated" else N, std=0.05, dtype=T)
    elif case["op"] == "linear":
        d["residual"] = normal(M, N, std=2.0, dtype=T) if case["residual"] else None
    return d


def prepare(case, seed):
    st = _draws(case, seed)
    st.update(case=case, T=TYPES[case["type"]])
    if case["op"] == "norm":
        # The stream after the block, which the backward pass reads and a training program has kept.
        if case["back"]:
            st["r"] = _plain_norm(st)["r"]
        if own:
            import paper_1602_02830_amd as bnn
            st["bnn"] = bnn
            st["kinds"] = {"none": bnn.NORM_NONE, "rms": bnn.NORM_RMS, "layer": bnn.NORM_LAYER}
            if not case["back"]:
                st["out_r"], st["out_n"] = torch.empty_like(st["y"]), torch.empty_like(st["y"]) if case["pre"] != "none" else None
            else:
                st["workspace"] = torch.empty(bnn.norm_residual_backward_workspace(case["M"], case["D"], case["rows_per_gate"]),
                                              dtype=torch.uint8, device=DEV)
        return st
    if own:
        import paper_1602_02830_amd as bnn
        st["bnn"] = bnn
        st["act"] = {"none": bnn.ACT_NONE, "relu": bnn.ACT_RELU, "silu": bnn.ACT_SILU, "gelu": bnn.ACT_GELU,
                     "gelu_tanh": bnn.ACT_GELU_TANH, "sigmoid": bnn.ACT_SIGMOID}[case["act"]]
        st["w_bits"] = bnn.pack_sign(st.pop("w"))
        M, K, n = case["M"], case["K"], case["F"] if case["op"] == "gated" else case["N"]
        if not case["back"]:
            st["out"] = torch.empty((M, n), dtype=st["T"], device=DEV)
        else:
            size = bnn.gated_bits_backward_workspace if case["op"] == "gated" else bnn.linear_bits_backward_workspace
            st["workspace"] = torch.empty(size(st["T"], M, n, K, st["act"]), dtype=torch.uint8, device=DEV)
    return st


# ---- the operators -----------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    if own:
        return _own_norm(st) if case["op"] == "norm" else _own_product(st)
    if case["op"] == "norm":
        return _plain_norm_back(st) if case["back"] else _plain_norm(st)
    return _plain_product_back(st) if case["back"] else _plain_product(st)


def _own_norm(st):
    bnn, case = st["bnn"], st["case"]
    post, pre = st["kinds"][case["post"]], st["kinds"][case["pre"]]
    if not case["back"]:
        r, n = bnn.norm_residual(st["y"], st["x"], st["gate"], st["res_scale"], post, st["post_gamma"], st["post_beta"],
                                 pre, st["pre_gamma"], st["pre_beta"], EPS, case["rows_per_gate"], out=st["out_r"], out_n=st["out_n"])
        return {"r": r, "n": n} if n is not None else {"r": r}
    got = bnn.norm_residual_backward(st["dr"], st["dn"], st["y"], st["r"], st["gate"], st["res_scale"], post, st["post_gamma"],
                                     st["post_beta"], pre, st["pre_gamma"], st["pre_beta"], EPS, case["rows_per_gate"],
                                     need_dx=case["x"], workspace=st["workspace"])
    return {k: v for k, v in got.items() if v is not None}


def _own_product(st):
    bnn, case = st["bnn"], st["case"]
    if case["op"] == "gated":
        if not case["back"]:
            return bnn.gated_bits(st["x"], st["w_bits"], st["scale"], st["bias"], st["act"], out=st["out"])
        got = bnn.gated_bits_backward(st["dy"], st["x"], st["w_bits"], st["scale"], st["bias"], st["act"], workspace=st["workspace"])
    else:
        if not case["back"]:
            return bnn.linear_bits(st["x"], st["w_bits"], st["scale"], st["bias"], st["act"], st["residual"], out=st["out"])
        got = bnn.linear_bits_backward(st["dy"], st["x"], st["w_bits"], st["scale"], st["bias"], st["act"], workspace=st["workspace"])
    return {k: v for k, v in got.items() if v is not None}


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ----------------------------------

def _act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_grad(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name in ("silu", "sigmoid"):
        s = 1 / (1 + torch.exp(-z))
        return s * (1 - s) if name == "sigmoid" else s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def _plain_z(st, x):
    """The products and the values before the activation."""
    s = x @ st["w"].t()
    z = s if st["scale"] is None else s * st["scale"]
    return s, z if st["bias"] is None else z + st["bias"]


def _plain_product(st):
    case, T = st["case"], st["T"]
    _, z = _plain_z(st, st["x"].float())
    if case["op"] == "gated":
        F = case["F"]
        return (_act(z[:, :F], case["act"]) * z[:, F:]).to(T)
    y = _act(z, case["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(T)


def _plain_product_back(st):
    case, T = st["case"], st["T"]
    x, dy = st["x"].float(), st["dy"].float()
    s, z = _plain_z(st, x)
    if case["op"] == "gated":
        F = case["F"]
        zg, zu = z[:, :F], z[:, F:]
        dz = torch.cat([dy * zu * _act_grad(zg, case["act"]), dy * _act(zg, case["act"])], dim=1)
    else:
        dz = dy * _act_grad(z, case["act"])
    ds = dz if st["scale"] is None else dz * st["scale"]
    out = {"dx": (ds @ st["w"]).to(T), "dw": (ds.t() @ x).to(T)}
    if st["scale"] is not None:
        out["dscale"] = (dz * s).sum(0)
    if st["bias"] is not None:
        out["dbias"] = dz.sum(0)
    return out


def _plain_hat(v, kind):
    """The normalised rows and the factor that they were divided by."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    inv = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * inv, inv


def _plain_side(v, kind, gamma, beta):
    if kind == "none":
        return v
    hat, _ = _plain_hat(v, kind)
    return hat * gamma if beta is None else hat * gamma + beta


def _rows_gate(st):
    case = st["case"]
    return st["gate"].float().repeat_interleave(case["rows_per_gate"], 0)[:case["M"]]


def _plain_norm(st):
    case, T = st["case"], st["T"]
    t = _plain_side(st["y"].float(), case["post"], st["post_gamma"], st["post_beta"])
    r = t * st["res_scale"]
    if st["gate"] is not None:
        r = r * _rows_gate(st)
    if st["x"] is not None:
        r = r + st["x"].float()
    out = {"r": r.to(T)}
    if case["pre"] != "none":
        out["n"] = _plain_side(r, case["pre"], st["pre_gamma"], st["pre_beta"]).to(T)
    return out


def _plain_side_back(d, v, kind, gamma):
    """From the gradient of a norm's result to those of its input and of its parameters."""
    hat, inv = _plain_hat(v, kind)
    dh = d * gamma
    dv = dh - hat * (dh * hat).mean(1, keepdim=True)
    if kind == "layer":
        dv = dv - dh.mean(1, keepdim=True)
    return dv * inv, (d * hat).sum(0), d.sum(0)


def _plain_norm_back(st):
    case, T = st["case"], st["T"]
    out = {}
    d = st["dr"].float()
    if case["pre"] != "none":
        more, dgamma, dbeta = _plain_side_back(st["dn"].float(), st["r"].float(), case["pre"], st["pre_gamma"])
        d = d + more
        out["dpre_gamma"] = dgamma
        if case["pre"] == "layer":
            out["dpre_beta"] = dbeta
    if case["x"]:
        out["dx"] = d.to(T)
    y = st["y"].float()
    dt = d * st["res_scale"]
    if st["gate"] is not None:
        R, M, D = case["rows_per_gate"], case["M"], case["D"]
        each = dt * _plain_side(y, case["post"], st["post_gamma"], st["post_beta"])
        G = -(-M // R)
        if G * R > M:
            each = torch.cat([each, each.new_zeros(G * R - M, D)])
        out["dgate"] = each.view(G, R, D).sum(1).to(T)
        dt = dt * _rows_gate(st)
    if case["post"] != "none":
        dt, dgamma, dbeta = _plain_side_back(dt, y, case["post"], st["post_gamma"])
        out["dpost_gamma"] = dgamma
        if case["post"] == "layer":
            out["dpost_beta"] = dbeta
    out["dy"] = dt.to(T)
    return out


# ---- what an operator cannot do without ----------------------------------------------------------------------

def work(case):
    size = BYTES[case["type"]]
    M = case["M"]
    if case["op"] == "norm":
        D, G = case["D"], -(-case["M"] // case["rows_per_gate"])
        sides = sum({"none": 0, "rms": 1, "layer": 2}[case[s]] for s in ("post", "pre"))
        if not case["back"]:
            b = size * M * D * (2 + case["x"] + (case["pre"] != "none")) + size * G * D * case["gate"] + 4 * D * sides
            return {"bytes": b, "flops": 12 * M * D}
        # dr, y and dy; with a norm of r: dn and r; dx
        b = size * M * D * (3 + 2 * (case["pre"] != "none") + case["x"]) + 2 * size * G * D * case["gate"] + 12 * D * sides
        return {"bytes": b, "flops": 30 * M * D}
    K, gated = case["K"], case["op"] == "gated"
    N, out = (2 * case["F"], case["F"]) if gated else (case["N"], case["N"])
    bits = 4 * N * ((K + 31) // 32)
    vectors = 4 * N * (case["scale"] + case["bias"])
    if not case["back"]:
        return {"bytes": size * (M * K + M * out * (1 + case.get("residual", False))) + bits + vectors, "flops": 2 * M * N * K}
    # Two products for the gradients; with an activation one more for the values that it was taken of.
    products = 2 if case["act"] == "none" and not gated else 3
    return {"bytes": size * (2 * M * K + M * out + N * K) + bits + 2 * vectors, "flops": products * 2 * M * N * K}


# ---- the same results from the definitions, in 64 bits -------------------------------------------------------

def _phi(z, name):
    """An activation and its derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        # 0.5 z (1 + tanh u) = z sigmoid(2 u)
        u2 = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        s = torch.sigmoid(u2)
        return z * s, s + z * s * (1 - s) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z ** 2)
    s = torch.sigmoid(z)
    if name == "sigmoid":
        return s, s * (1 - s)
    return z * s, s + z * s * (1 - s)


def _exact_product(case, d):
    x, w = d["x"].double(), d["w"].double()
    a = d["scale"].double() if d["scale"] is not None else torch.ones(w.shape[0], dtype=torch.float64, device=DEV)
    b = d["bias"].double() if d["bias"] is not None else torch.zeros(w.shape[0], dtype=torch.float64, device=DEV)
    s = torch.mm(x, w.t())
    z = torch.addcmul(b, s, a)
    if case["op"] == "gated":
        zg, zu = z.chunk(2, dim=1)
        f, df = _phi(zg, case["act"])
        if not case["back"]:
            return f.mul_(zu)
        dh = d["dy"].double()
        dz = torch.empty_like(z)
        dz[:, :case["F"]] = df.mul_(zu).mul_(dh)
        dz[:, case["F"]:] = f.mul_(dh)
        del zg, zu, f, df, dh
    else:
        f, df = _phi(z, case["act"])
        if not case["back"]:
            return f if d["residual"] is None else f + d["residual"].double()
        dz = df * d["dy"].double()
        del f, df
    del z
    out = {}
    if d["scale"] is not None:
        out["dscale"] = torch.einsum("mn,mn->n", dz, s)
    del s
    if d["bias"] is not None:
        out["dbias"] = dz.sum(dim=0)
    dz.mul_(a)
    out["dx"] = torch.mm(dz, w)
    out["dw"] = torch.mm(dz.t(), x)
    return {k: out[k] for k in ("dx", "dw", "dscale", "dbias") if k in out}


def _exact_norm_of(v, kind, gamma, beta):
    """A norm's result and what its derivative needs."""
    if kind == "none":
        return v, None
    centre = v.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros(v.shape[0], 1, dtype=torch.float64, device=DEV)
    sigma = torch.sqrt(((v - centre) ** 2).mean(dim=1, keepdim=True) + EPS)
    hat = (v - centre) / sigma
    res = hat * gamma.double()
    return (res if beta is None else res + beta.double()), (hat, sigma)


def _exact_norm_grad(up, kept, kind, gamma):
    hat, sigma = kept
    q = up * gamma.double()
    inner = q - hat * (q * hat).mean(dim=1, keepdim=True)
    if kind == "layer":
        inner = inner - q.mean(dim=1, keepdim=True)
    return inner / sigma


def _exact_norm(case, d, r_kept):
    M, D, R = case["M"], case["D"], case["rows_per_gate"]
    y = d["y"].double()
    t, kept = _exact_norm_of(y, case["post"], d["post_gamma"], d["post_beta"])
    which = torch.arange(M, device=DEV) // R
    g = d["gate"].double()[which] if d["gate"] is not None else None
    if not case["back"]:
        r = d["res_scale"] * (t if g is None else g * t)
        if d["x"] is not None:
            r = r + d["x"].double()
        if case["pre"] == "none":
            return {"r": r}
        return {"r": r, "n": _exact_norm_of(r, case["pre"], d["pre_gamma"], d["pre_beta"])[0]}
    out = {}
    total = d["dr"].double()
    if case["pre"] != "none":
        dn = d["dn"].double()
        _, kept_r = _exact_norm_of(r_kept.double(), case["pre"], d["pre_gamma"], d["pre_beta"])
        total = total + _exact_norm_grad(dn, kept_r, case["pre"], d["pre_gamma"])
        out["dpre_gamma"] = (dn * kept_r[0]).sum(dim=0)
        if case["pre"] == "layer":
            out["dpre_beta"] = dn.sum(dim=0)
    if case["x"]:
        out["dx"] = total
    up = d["res_scale"] * total
    if g is not None:
        out["dgate"] = torch.zeros(d["gate"].shape, dtype=torch.float64, device=DEV).index_add_(0, which, up * t)
        up = up * g
    if case["post"] != "none":
        out["dpost_gamma"] = (up * kept[0]).sum(dim=0)
        if case["post"] == "layer":
            out["dpost_beta"] = up.sum(dim=0)
        up = _exact_norm_grad(up, kept, case["post"], d["post_gamma"])
    out["dy"] = up
    return out


def exact(case, seed):
    d = _draws(case, seed)
    if case["op"] != "norm":
        return _exact_product(case, d)
    r = None
    if case["back"] and case["pre"] != "none":
        r = _plain_norm({**d, "case": case, "T": TYPES[case["type"]]})["r"]      # an input of the backward pass
    return _exact_norm(case, d, r)
