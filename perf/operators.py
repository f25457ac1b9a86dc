"""Performance cases of the operators around a transformer block's linears:
4-bit microscaled (MXFP4) weights and activations, the gated feed-forward and
rotary positions, each in a plain form and through the public entry points of
`paper_2607_08526_amd.qlinear`.

    own                 False: `run` computes the plain form; True: it calls
                        the library
    listed()            the cases themselves
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs and weights of one case
    run(state)          one pass; returns every output whole
    work(case)          bytes and flops a pass cannot do without
    exact(case, seed)   the outputs in 64 bits, from the definition

Kinds of case:

  quant    MXFP4 codes and scales of a tensor, and the tensor read back from
           them: a weight at load time, or a layer's activations
  product  a linear layer with MXFP4 weights through its epilogue; x names the
           activations: bf16, f32, or mx (bf16 activations that the pass
           quantizes to MXFP4 first, for the 4-bit matrix cores)
  gated    H = act(X Wg^T + bg) * (X Wu^T + bu): the first half of a gated
           feed-forward block
  grad     the backward pass of gated: the gradient of X and, with dw, of both
           weights
  rotary   rotary positions of the query and key heads of a fused QKV tensor

MXFP4: blocks of 32 values along a row share a scale 2^(s - 127), s one byte;
a value is a sign, and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6.  Weights
are N(0, 0.02) and activations N(0, 1), as in synth_inputs.py; normalised
activations have a few large channels, and those here do too.
"""
import math

import torch

own = False

BLOCK = 32
QMAX = {"q4": 7, "int8": 127}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # the smallest: one clip's conditioning rows, a ragged count, on their
        # way into a 4-bit product
        {"name": "quant activations", "kind": "quant", "x": "bf16", "M": 13, "K": 1536},
        # load time: one FFN-up weight
        {"name": "quant weight", "kind": "quant", "x": "weight", "M": 8192, "K": 2048},
        # few rows: a single token's FFN-up layer of the d = 1536 model
        {"name": "product 1 row", "kind": "product", "x": "bf16", "M": 1, "N": 6144, "K": 1536,
         "ep": "gelu"},
        # an odd layer on fp32 activations (a conditioning projection)
        {"name": "product f32 odd", "kind": "product", "x": "f32", "M": 77, "N": 1000, "K": 1056,
         "ep": "none"},
        # a batch of 2048 tokens through the FFN-up layer of the d = 2048 model
        {"name": "product 2048 rows", "kind": "product", "x": "bf16", "M": 2048, "N": 8192,
         "K": 2048, "ep": "gelu"},
        # two guidance branches of a 60 s clip in 4-bit arithmetic, d = 1536
        {"name": "product mx 60 s", "kind": "product", "x": "mx", "M": 1290, "N": 6144,
         "K": 1536, "ep": "full"},
        # a single token through the gated feed-forward of the d = 1536 model
        {"name": "gated 1 row", "kind": "gated", "fmt": "mxfp4", "M": 1, "N": 4096, "K": 1536,
         "act": "silu", "bias": False},
        # a batch of 2048 tokens, d = 2048, hidden width 8/3 d rounded up to 64
        {"name": "gated 2048 rows", "kind": "gated", "fmt": "mxfp4", "M": 2048, "N": 5504,
         "K": 2048, "act": "silu", "bias": True},
        # adapters on frozen 4-bit weights: one 10 s clip, the gradient of X
        {"name": "grad q4 clip", "kind": "grad", "fmt": "q4", "M": 107, "N": 2752, "K": 1024,
         "act": "gelu", "bias": False, "dw": False},
        # the largest: quantization-aware training of the d = 1536 model, the
        # gradients of X and of both weights
        {"name": "grad mxfp4 2048 rows", "kind": "grad", "fmt": "mxfp4", "M": 2048, "N": 4096,
         "K": 1536, "act": "silu", "bias": True, "dw": True},
        # one far token of a stream, neighbouring channels in pairs
        {"name": "rotary 1 token", "kind": "rotary", "x": "f32", "B": 1, "T": 1, "H": 32,
         "rot": 64, "layout": "interleaved", "far": True, "adjoint": False},
        # two sequences of 4096 tokens, d = 2048, half of each head rotated
        {"name": "rotary 8192 tokens", "kind": "rotary", "x": "bf16", "B": 2, "T": 4096, "H": 32,
         "rot": 32, "layout": "half", "far": False, "adjoint": False},
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], uniform in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A reduction length: whole 256-column widths as in the models, or any
    multiple of a block."""
    if rng.random() < 0.6:
        return 256 * _log(rng, max(1, lo // 256), hi // 256)
    return BLOCK * _log(rng, lo // BLOCK, hi // BLOCK)


def draw(rng):
    kind = rng.choice(["quant", "product", "product", "gated", "gated", "grad", "grad",
                       "rotary"])
    if kind == "quant":
        return {"kind": kind, "x": rng.choice(["bf16", "f32", "weight"]), "M": _log(rng, 1, 8192),
                "K": BLOCK * _log(rng, 1, 64)}
    if kind == "product":
        return {"kind": kind, "x": rng.choice(["bf16", "bf16", "f32", "mx", "mx"]),
                "M": _log(rng, 1, 2100), "N": _log(rng, 64, 8200), "K": _width(rng, 256, 2048),
                "ep": rng.choice(["none", "bias", "gelu", "full"])}
    if kind in ("gated", "grad"):
        case = {"kind": kind, "fmt": rng.choice(["mxfp4", "mxfp4", "q4", "int8"]),
                "M": _log(rng, 1, 2048), "N": _log(rng, 128, 4096),
                "K": _width(rng, 256, 1536), "act": rng.choice(["silu", "gelu"]),
                "bias": rng.random() < 0.5}
        if kind == "grad":  # N is the next layer's reduction length
            case["N"] = 8 * (case["N"] // 8)
            case["dw"] = rng.random() < 0.5
        return case
    return {"kind": kind, "x": rng.choice(["bf16", "f32"]), "B": rng.randint(1, 2),
            "T": _log(rng, 1, 2048), "H": rng.randint(4, 32), "rot": rng.choice([16, 32, 48, 64]),
            "layout": rng.choice(["half", "interleaved"]), "far": rng.random() < 0.5,
            "adjoint": rng.random() < 0.3}


# ---- inputs (shared by prepare and exact: the same seed, the same values) ----

class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device="cuda") * std

    def activations(self, M, K):
        """Rows of N(0, 1) with one channel in 64 ten times as large."""
        big = 1.0 + 9.0 * (torch.rand(K, generator=self.g, device="cuda") < 1 / 64)
        return self.normal(M, K) * big


def _dtype(x):
    return torch.float32 if x in ("f32", "weight") else torch.bfloat16


def _quant_inputs(case, seed):
    r = _Draw(seed)
    M, K = case["M"], case["K"]
    if case["x"] == "weight":
        return r.normal(M, K, std=0.02)
    return r.activations(M, K).to(_dtype(case["x"]))


def _product_inputs(case, seed):
    r = _Draw(seed)
    M, N, K, ep = case["M"], case["N"], case["K"], case["ep"]
    codes, scales = _pack_mx(*_plain_mx(r.normal(N, K, std=0.02)))
    return (r.activations(M, K).to(_dtype(case["x"])), codes, scales,
            r.normal(N, std=0.1) if ep != "none" else None,
            r.normal(M, N) if ep == "full" else None)


def _gated_inputs(case, seed):
    r = _Draw(seed)
    M, N, K, fmt = case["M"], case["N"], case["K"], case["fmt"]
    gate, up = (_pack(fmt, r.normal(N, K, std=1 / math.sqrt(K))) for _ in range(2))
    X = r.normal(M, K).to(torch.bfloat16)
    bias = (r.normal(N, std=0.1), r.normal(N, std=0.1)) if case["bias"] else None
    dH = r.normal(M, N, std=0.05).to(torch.bfloat16) if case["kind"] == "grad" else None
    return X, gate, up, bias, dH


def _rotary_inputs(case, seed):
    r = _Draw(seed)
    rows, heads = case["B"] * case["T"], case["H"]
    qkv = r.normal(rows, 3 * heads * 64).to(_dtype(case["x"]))
    # positions of each sequence: from its start, or after a long past
    start = torch.randint(0, 1 << 20 if case["far"] else 1, (case["B"], 1), generator=r.g,
                          device="cuda")
    positions = (start + torch.arange(case["T"], device="cuda")).reshape(-1)
    # radians per position, base 10000, slowed fourfold for a longer context
    freqs = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device="cuda") /
                        case["rot"]) / 4.0
    return qkv, positions, freqs, 0.1 * math.log(4.0) + 1.0


# ---- the plain forms -------------------------------------------------------

def _plain_mx(x):
    """(codes, scale bytes) of x in blocks of 32: the scale is the power of two
    that puts the largest magnitude of a block into [4, 8), the codes are the
    nearest magnitudes (ties to the even code, 6 for what is beyond), bit 3
    the sign."""
    b = x.float().reshape(x.shape[0], -1, BLOCK)
    top = torch.frexp(b.abs().amax(dim=2))[1] - 3
    top = torch.where(b.abs().amax(dim=2) == 0, -127, top).clamp(-127, 127)
    v = torch.ldexp(b.double(), -top.unsqueeze(2)).abs()
    code = sum((v >= t if i % 2 else v > t).to(torch.uint8)
               for i, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)))
    code = code + 8 * torch.signbit(b).to(torch.uint8)
    return code.reshape(x.shape), (top + 127).to(torch.uint8)


def _pack_mx(codes, scales):
    return codes[:, ::2] | codes[:, 1::2] << 4, scales


def _pack(fmt, W):
    """(codes, scales) of a weight as the library lays them out."""
    if fmt == "mxfp4":
        return _pack_mx(*_plain_mx(W))
    q = QMAX[fmt]
    b = W.double().reshape(W.shape[0], -1, BLOCK)
    s = (b.abs().amax(dim=2) / q).to(torch.float16)
    c = (b / s.double().unsqueeze(2)).round().clamp(-q, q).to(torch.int8).reshape(W.shape)
    s = s.view(torch.int16)
    if fmt == "int8":
        return c.view(torch.uint8), s
    c = c.view(torch.uint8) & 15
    return c[:, ::2] | c[:, 1::2] << 4, s


def _plain_values(fmt, codes, scales):
    """The fp32 values that codes and scales stand for."""
    if fmt == "int8":
        v = codes.view(torch.int8).float()
    else:
        c = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1).long()
        if fmt == "mxfp4":
            table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
            v = table[c]
        else:
            v = (c - 16 * (c >= 8)).float()
    b = v.reshape(v.shape[0], -1, BLOCK)
    if fmt == "mxfp4":
        b = torch.ldexp(b, scales.int().unsqueeze(2) - 127)
    else:
        b = b * scales.view(torch.float16).float().unsqueeze(2)
    return b.reshape(v.shape)


def _plain_gelu(x):
    return x * (1 + torch.erf(x / math.sqrt(2))) / 2


def _plain_act(act, x):
    """act(x) and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-x))
        return x * s, s * (1 + x * (1 - s))
    phi = (1 + torch.erf(x / math.sqrt(2))) / 2
    return x * phi, phi + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def _plain_quant(s):
    return _plain_values("mxfp4", *_pack_mx(*_plain_mx(s["X"]))).to(s["X"].dtype)


def _plain_product(s):
    X = s["X"].float()
    if s["x"] == "mx":
        X = _plain_values("mxfp4", *_pack_mx(*_plain_mx(X)))
    Y = X @ _plain_values("mxfp4", s["codes"], s["scales"]).t()
    if s["bias"] is not None:
        Y = Y + s["bias"]
    if s["ep"] == "gelu":
        Y = _plain_gelu(Y)
    if s["residual"] is not None:
        Y = Y + s["residual"]
    return Y.to(s["ydtype"])


def _plain_gated(s):
    X = s["X"].float()
    Wg, Wu = (_plain_values(s["fmt"], *w) for w in (s["gate"], s["up"]))
    G, U = X @ Wg.t(), X @ Wu.t()
    if s["bias"] is not None:
        G, U = G + s["bias"][0], U + s["bias"][1]
    a, da = _plain_act(s["act"], G)
    if s["dH"] is None:
        return (a * U).to(torch.bfloat16)
    dH = s["dH"].float()
    dG, dU = dH * U * da, dH * a
    out = [(dG @ Wg + dU @ Wu).to(torch.bfloat16)]
    if s["dw"]:
        out += [(d.t() @ X).to(torch.bfloat16) for d in (dG, dU)]
    return out


def _plain_rotary(s):
    rows, H, rot = s["X"].shape[0], 2 * s["H"], s["rot"]
    x = s["X"].float().reshape(rows, H, 64)
    angle = s["positions"].double().unsqueeze(1) * s["freqs"]
    cos = (torch.cos(angle) * s["mscale"]).float().unsqueeze(1)
    sin = (torch.sin(angle) * s["mscale"]).float().unsqueeze(1)
    sin = -sin if s["adjoint"] else sin
    if s["layout"] == "half":
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=3).flatten(2)
    return torch.cat((turned, x[..., rot:]), dim=2).reshape(rows, -1).to(s["X"].dtype)


# ---- the library's calls ----------------------------------------------------

def _own_quant(s):
    from paper_2607_08526_amd import qlinear as ql
    codes, scales = ql.quantize(ql.FMT_MXFP4, s["X"]) if s["x"] == "weight" \
        else ql.quantize_act_mx(s["X"])
    return ql.dequantize(ql.FMT_MXFP4, codes, scales, dtype=s["X"].dtype)


def _own_product(s):
    from paper_2607_08526_amd import qlinear as ql
    N = s["codes"].shape[0]
    ep = dict(bias=s["bias"], act=ql.ACT_GELU if s["ep"] == "gelu" else ql.ACT_NONE,
              residual=s["residual"], ydtype=s["ydtype"])
    if s["x"] == "mx":
        qx, sx = ql.quantize_act_mx(s["X"])
        return ql.forward_mx(qx, sx, s["codes"], s["scales"], N, **ep)
    return ql.forward_ep(ql.FMT_MXFP4, s["X"], s["codes"], s["scales"], N, **ep)


def _own_gated(s):
    from paper_2607_08526_amd import qlinear as ql
    fmt = {"mxfp4": ql.FMT_MXFP4, "q4": ql.FMT_Q4, "int8": ql.FMT_INT8}[s["fmt"]]
    act = {"silu": ql.ACT_SILU, "gelu": ql.ACT_GELU}[s["act"]]
    if s["dH"] is None:
        return ql.gated_forward(fmt, s["X"], s["gate"], s["up"], bias=s["bias"], act=act)
    g = ql.gated_backward(fmt, s["X"], s["gate"], s["up"], s["dH"], bias=s["bias"], act=act,
                          weight_grads=s["dw"])
    return [g.X, g.W_gate, g.W_up] if s["dw"] else [g.X]


def _own_rotary(s):
    from paper_2607_08526_amd import qlinear as ql
    return ql.rotary(s["X"], 2 * s["H"], s["freqs"], positions=s["positions"],
                     interleaved=s["layout"] == "interleaved", mscale=s["mscale"],
                     adjoint=s["adjoint"], out=s["out"])


# ---- prepare and run -------------------------------------------------------

def prepare(case, seed):
    kind = case["kind"]
    if kind == "quant":
        return {"kind": kind, "x": case["x"], "X": _quant_inputs(case, seed)}
    if kind == "product":
        X, codes, scales, bias, residual = _product_inputs(case, seed)
        return {"kind": kind, "x": case["x"], "ep": case["ep"], "X": X, "codes": codes,
                "scales": scales, "bias": bias, "residual": residual,
                "ydtype": torch.bfloat16 if case["ep"] == "gelu" else torch.float32}
    if kind in ("gated", "grad"):
        X, gate, up, bias, dH = _gated_inputs(case, seed)
        return {"kind": kind, "fmt": case["fmt"], "act": case["act"], "X": X, "gate": gate,
                "up": up, "bias": bias, "dH": dH, "dw": case.get("dw", False)}
    qkv, positions, freqs, mscale = _rotary_inputs(case, seed)
    X = qkv[:, : 2 * case["H"] * 64]
    return {"kind": kind, "X": X, "H": case["H"], "rot": case["rot"], "layout": case["layout"],
            "adjoint": case["adjoint"], "positions": positions, "freqs": freqs, "mscale": mscale,
            "out": torch.empty(X.shape, dtype=X.dtype, device=X.device)}


def run(state):
    form = {"quant": (_plain_quant, _own_quant), "product": (_plain_product, _own_product),
            "gated": (_plain_gated, _own_gated), "grad": (_plain_gated, _own_gated),
            "rotary": (_plain_rotary, _own_rotary)}
    return form[state["kind"]][1 if own else 0](state)


def _weight_bytes(fmt, N, K):
    if fmt == "mxfp4":
        return N * K // 2 + N * K // BLOCK
    return N * K // (2 if fmt == "q4" else 1) + N * K // BLOCK * 2


def work(case):
    kind = case["kind"]
    if kind == "quant":
        M, K = case["M"], case["K"]
        size = 2 if case["x"] == "bf16" else 4
        return {"bytes": 2 * M * K * size, "flops": 2 * M * K}
    if kind == "rotary":
        rows, heads = case["B"] * case["T"], 2 * case["H"]
        size = 2 if case["x"] == "bf16" else 4
        return {"bytes": 2 * rows * heads * 64 * size + 8 * rows + 4 * case["rot"],
                "flops": 3 * rows * heads * case["rot"]}
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "product":
        ep = case["ep"]
        return {"bytes": M * K * (4 if case["x"] == "f32" else 2) + _weight_bytes("mxfp4", N, K)
                + M * N * (2 if ep == "gelu" else 4) + (4 * N if ep != "none" else 0)
                + (4 * M * N if ep == "full" else 0), "flops": 2 * M * N * K}
    both = 2 * _weight_bytes(case["fmt"], N, K) + (8 * N if case["bias"] else 0)
    bytes_, flops = 2 * M * K + both + 2 * M * N, 4 * M * N * K
    if kind == "grad":  # X's gradient, and the weights'
        bytes_, flops = bytes_ + 2 * M * K, 2 * flops
        if case["dw"]:
            bytes_, flops = bytes_ + 4 * N * K, flops + 4 * M * N * K
    return {"bytes": bytes_, "flops": flops}


# ---- the operators in 64 bits ------------------------------------------------

def _exact_mx(x):
    """x as MXFP4 values, from the definition: round to the spacing of the
    binade that x / scale lies in."""
    b = x.double().reshape(x.shape[0], -1, BLOCK)
    top = b.abs().amax(dim=2, keepdim=True)
    e = torch.floor(torch.log2(top))
    # log2 may round to the next integer just below a power of two
    e = torch.where(torch.exp2(e) > top, e - 1, torch.where(torch.exp2(e + 1) <= top, e + 1, e))
    scale = torch.exp2((e - 2).clamp(-127, 127))
    v = b / scale
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0))
    q = (torch.round(v / step) * step).clamp(-6, 6)
    return torch.where(top == 0, 0.0, q * scale).reshape(x.shape)


def _exact_weight(fmt, codes, scales):
    """The 64-bit values of codes and scales, from their bit fields."""
    if fmt == "int8":
        c = codes.to(torch.float64)
        v = torch.where(c >= 128, c - 256, c)
    else:
        nib = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.int64,
                          device=codes.device)
        nib[:, 0::2], nib[:, 1::2] = codes % 16, codes // 16
        if fmt == "q4":
            v = nib.double() - 16.0 * (nib > 7)
        else:
            exponent, mantissa = nib // 2 % 4, (nib % 2).double()
            v = torch.where(exponent == 0, mantissa / 2,
                            (1 + mantissa / 2) * torch.exp2(exponent.double() - 1))
            v = torch.where(nib > 7, -v, v)
    s = torch.exp2(scales.double() - 127) if fmt == "mxfp4" \
        else scales.view(torch.float16).double()
    return v * s.repeat_interleave(BLOCK, dim=1)


def exact(case, seed):
    kind = case["kind"]
    if kind == "quant":
        return _exact_mx(_quant_inputs(case, seed))
    if kind == "product":
        X, codes, scales, bias, residual = _product_inputs(case, seed)
        X = _exact_mx(X) if case["x"] == "mx" else X.double()
        Y = torch.mm(X, _exact_weight("mxfp4", codes, scales).T.contiguous())
        if bias is not None:
            Y += bias.double()
        if case["ep"] == "gelu":
            Y = Y * torch.special.ndtr(Y)
        return Y if residual is None else Y + residual.double()
    if kind in ("gated", "grad"):
        X, gate, up, bias, dH = _gated_inputs(case, seed)
        X, Wg, Wu = X.double(), _exact_weight(case["fmt"], *gate), _exact_weight(case["fmt"], *up)
        bg, bu = (0.0, 0.0) if bias is None else (b.double() for b in bias)
        leaves = [t.requires_grad_(kind == "grad") for t in (X, Wg, Wu)]
        G, U = torch.mm(X, Wg.T) + bg, torch.mm(X, Wu.T) + bu
        H = G * (torch.sigmoid(G) if case["act"] == "silu" else torch.special.ndtr(G)) * U
        if kind == "gated":
            return H
        grads = torch.autograd.grad(H, leaves if case["dw"] else leaves[:1], dH.double())
        return list(grads)
    qkv, positions, freqs, mscale = _rotary_inputs(case, seed)
    rows, H, rot = qkv.shape[0], 2 * case["H"], case["rot"]
    x = qkv[:, : H * 64].double().reshape(rows, H, 64)
    t = positions.double()[:, None] * freqs * (-1.0 if case["adjoint"] else 1.0)
    turn = torch.polar(torch.full_like(t, mscale), t)[:, None, :]
    at = torch.arange(rot, device=x.device)
    first, second = at.reshape(2, -1) if case["layout"] == "half" else at.reshape(-1, 2).T
    z = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return x.reshape(rows, -1)
