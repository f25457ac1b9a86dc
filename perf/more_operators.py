"""Performance cases of the normalisation and the masked attention of a
transformer block, with their backward passes, each in a plain form and through
the public entry points of `paper_2607_08526_amd.qlinear`.

    own                 False: `run` computes the plain form; True: it calls
                        the library
    listed()            the cases themselves
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs of one case
    run(state)          one pass; returns every output whole
    work(case)          bytes and flops a pass cannot do without
    exact(case, seed)   the outputs in 64 bits, from the definition

Kinds of case:

  norm       h = x + residual, y = w h / sqrt(mean(h^2) + eps): a block's
             normalisation with the residual's addition; y in bf16, or as the
             int8 activations of an 8-bit product (returned as their values)
  norm_grad  its backward pass: the gradient of h (to x and to the residual
             alike, with the one that arrives at h added) and that of w
  attend     softmax attention; H query heads share Hk key heads; causal: query
             i of T sees the keys up to i + kT - T; rows says where sequences
             lie: full (all of the same length), padded (in T rows each, with
             their lengths) or packed (one behind the other, by offsets)
  train      the same forward and backward: the output, the logarithms of the
             row sums, and the gradients of q, k and v

Sizes are those of the d = 1024, 1536 and 2048 models (heads of 64) and of
their clips (107 tokens for 10 s, 645 for 60 s), and generic ones.
"""
import math
import random

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # the smallest: a single token of a stream, d = 1536, the fp32 residual
        # stream and a linear layer's bf16 output
        {"name": "norm 1 token", "kind": "norm", "M": 1, "N": 1536, "x": "bf16", "h": "f32",
         "y": "bf16", "w": True},
        # a batch of 2048 tokens, d = 2048
        {"name": "norm 2048 rows", "kind": "norm", "M": 2048, "N": 2048, "x": "f32", "h": "f32",
         "y": "bf16", "w": True},
        # two guidance branches of a 60 s clip on the way into an 8-bit product
        {"name": "norm int8 60 s", "kind": "norm", "M": 1290, "N": 1536, "x": "bf16", "h": "f32",
         "y": "int8", "w": True},
        # training on one 10 s clip, d = 1024
        {"name": "norm grad clip", "kind": "norm_grad", "M": 107, "N": 1024, "x": "bf16",
         "h": "f32", "dx": "f32", "w": True},
        # training on 8192 tokens, d = 2048
        {"name": "norm grad 8192 rows", "kind": "norm_grad", "M": 8192, "N": 2048, "x": "bf16",
         "h": "f32", "dx": "f32", "w": True},
        # a new token of eight requests over their caches of up to 8192 keys
        {"name": "attend 1 token", "kind": "attend", "B": 8, "T": 1, "kT": 8192, "H": 32, "Hk": 8,
         "dh": 128, "causal": False, "rows": "padded"},
        # a 60 s clip's tokens attend to a few conditioning rows, d = 1536
        {"name": "attend cross", "kind": "attend", "B": 2, "T": 645, "kT": 77, "H": 24, "Hk": 24,
         "dh": 64, "causal": False, "rows": "packed"},
        # two long sequences, d = 2048
        {"name": "attend causal 4096", "kind": "attend", "B": 2, "T": 4096, "kT": 4096, "H": 32,
         "Hk": 32, "dh": 64, "causal": True, "rows": "full"},
        # two 10 s clips, d = 1536
        {"name": "train clip", "kind": "train", "B": 2, "T": 107, "kT": 107, "H": 24, "Hk": 24,
         "dh": 64, "causal": False, "rows": "full"},
        # a batch of clips of unlike lengths, one behind the other, d = 2048
        {"name": "train packed clips", "kind": "train", "B": 5, "T": 645, "kT": 645, "H": 32,
         "Hk": 32, "dh": 64, "causal": False, "rows": "packed"},
        # causal training with four query heads to a key head
        {"name": "train causal 2048", "kind": "train", "B": 1, "T": 2048, "kT": 2048, "H": 32,
         "Hk": 8, "dh": 128, "causal": True, "rows": "full"},
        # the largest: a long sequence, d = 2048
        {"name": "train 4096", "kind": "train", "B": 1, "T": 4096, "kT": 4096, "H": 32, "Hk": 32,
         "dh": 64, "causal": False, "rows": "full"},
    ]


def _log(rng, lo, hi):
    """An integer in [lo, hi], uniform in its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "attend", "attend", "train", "train"])
    if kind in ("norm", "norm_grad"):
        case = {"kind": kind, "M": _log(rng, 1, 8192), "N": _log(rng, 33, 2048),
                "x": rng.choice(["bf16", "bf16", "f32"]), "h": rng.choice(["f32", "f32", "bf16"]),
                "w": rng.random() < 0.8}
        if kind == "norm_grad":
            return {**case, "dx": rng.choice(["f32", "bf16"])}
        case["y"] = rng.choice(["bf16", "f32", "int8"])
        if case["y"] == "int8" or rng.random() < 0.5:  # whole blocks of a weight
            case["N"] = 32 * max(1, case["N"] // 32)
        return case
    dh, Hk, group = rng.choice([64, 64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4])
    case = {"kind": kind, "H": Hk * group, "Hk": Hk, "dh": dh}
    if kind == "attend" and rng.random() < 0.5:  # few queries at the end of long caches
        T = _log(rng, 1, 16)
        return {**case, "B": rng.randint(1, 8), "T": T, "kT": _log(rng, 16, 16384),
                "causal": T > 1, "rows": rng.choice(["full", "padded"])}
    B, T = rng.randint(1, 4), _log(rng, 1, 2048)
    while B * T * T * case["H"] * dh > 4096 * 4096 * 32 * 64:  # no more than the largest listed
        B -= 1
    if rng.random() < 0.25:  # attention to other rows
        return {**case, "B": B, "T": T, "kT": _log(rng, 1, 1024), "causal": False,
                "rows": rng.choice(["full", "padded", "packed"])}
    return {**case, "B": B, "T": T, "kT": T, "causal": rng.random() < 0.5,
            "rows": rng.choice(["full", "padded", "packed"])}


# ---- inputs (shared by prepare and exact: the same seed, the same values) ----

def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape, std=1.0):
        return torch.randn(shape, generator=self.g, device="cuda") * std

    def stream(self, M, N):
        """A residual stream's rows: one channel in 64 ten times as large."""
        big = 1.0 + 9.0 * (torch.rand(N, generator=self.g, device="cuda") < 1 / 64)
        return self.normal(M, N) * big


def _norm_inputs(case, seed):
    r = _Draw(seed)
    M, N = case["M"], case["N"]
    weight = 1.0 + r.normal(N, std=0.2) if case["w"] else None
    if case["kind"] == "norm":
        return r.normal(M, N).to(_dtype(case["x"])), r.stream(M, N).to(_dtype(case["h"])), weight
    return (r.normal(M, N, std=0.05).to(_dtype(case["x"])), r.stream(M, N).to(_dtype(case["h"])),
            weight, r.normal(M, N, std=0.05).to(_dtype(case["dx"])))


def _lengths(B, T):
    """Lengths of B sequences, from T down to about half of it."""
    return [max(1, T - T * b // (2 * B)) for b in range(B)]


def _rows(case, keys, order):
    """(rows of the tensor, first rows, lengths) of the sequences of one side."""
    B, T = case["B"], case["kT" if keys else "T"]
    rows = case["rows"] if keys or case["T"] == case["kT"] else "full"
    lens = [T] * B if rows == "full" else [_lengths(B, T)[i] for i in order]
    if rows != "packed":
        return B * T, [b * T for b in range(B)], lens
    # buffers of whole 64 rows: those behind the last sequence belong to none
    first = [sum(lens[:b]) for b in range(B)]
    return -(-sum(lens) // 64) * 64, first, lens


def _attend_inputs(case, seed):
    r = _Draw(seed)
    order = list(range(case["B"]))
    random.Random(seed).shuffle(order)
    (qrows, qfirst, qlens), (krows, kfirst, klens) = (_rows(case, s, order) for s in (0, 1))
    wide, narrow = case["H"] * case["dh"], case["Hk"] * case["dh"]
    bf = lambda t: t.to(torch.bfloat16)
    if case["T"] == case["kT"]:  # the columns of a fused QKV output
        qkv = bf(r.normal(qrows, wide + 2 * narrow))
        q, k, v = qkv.split([wide, narrow, narrow], dim=1)
    else:
        q, k, v = bf(r.normal(qrows, wide)), bf(r.normal(krows, narrow)), bf(r.normal(krows, narrow))
    dO = bf(r.normal(qrows, wide, std=0.05)) if case["kind"] == "train" else None
    return q, k, v, dO, (qfirst, qlens), (kfirst, klens)


# ---- the plain forms -------------------------------------------------------

def _plain_norm(s):
    v = s["x"].float() + s["residual"].float()
    h = v.to(s["residual"].dtype)
    if s["y"] != "int8":
        y = v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
        return (y if s["weight"] is None else y * s["weight"]).to(_dtype(s["y"])), h
    # codes are nearest integers: values next to a border, in 64 bits
    v = v.double()
    y = v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    y = (y if s["weight"] is None else y * s["weight"].double()).float().double()
    scale = (y.abs().amax(dim=1, keepdim=True) / 127).to(torch.float16).double()
    codes = torch.round(y / scale).clamp(-127, 127)
    return (codes * scale).to(torch.bfloat16), h


def _plain_norm_grad(s):
    h, dy, N = s["h"].float(), s["dy"].float(), s["h"].shape[1]
    rstd = torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS)
    unit = h * rstd
    g = dy if s["weight"] is None else dy * s["weight"]
    dx = s["dres"].float() + rstd * (g - unit * ((g * unit).sum(dim=1, keepdim=True) / N))
    return dx.to(s["dres"].dtype), None if s["weight"] is None else (dy * unit).sum(dim=0)


def _plain_gather(x, heads, at, live):
    """[B, heads, T, dh] in fp32 of rows, zeros where no row is live."""
    rows = x[at.clamp(max=x.shape[0] - 1)].float() * live.unsqueeze(2)
    return rows.unflatten(2, (heads, -1)).transpose(1, 2).contiguous()


def _plain_scatter(x, at, live, rows, dtype):
    """The rows of [B, heads, T, dh] back where they came from, zeros elsewhere."""
    out = torch.zeros((rows + 1, x.shape[1] * x.shape[3]), device=x.device)
    out[torch.where(live, at, rows)] = x.transpose(1, 2).flatten(2)
    return out[:rows].to(dtype)


def _plain_attend(s):
    H, Hk, T, kT, scale = s["H"], s["Hk"], s["T"], s["kT"], s["dh"] ** -0.5
    t, j = torch.arange(T, device="cuda"), torch.arange(kT, device="cuda")
    qat, kat = s["qfirst"].unsqueeze(1) + t, s["kfirst"].unsqueeze(1) + j
    qlens, klens = s["qlens"].unsqueeze(1), s["klens"].unsqueeze(1)
    qlive, klive = t < qlens, j < klens
    q = _plain_gather(s["q"], H, qat, qlive)
    k, v = (_plain_gather(s[n], Hk, kat, klive).repeat_interleave(H // Hk, dim=1) for n in "kv")
    mask = qlive.unsqueeze(2) & klive.unsqueeze(1)
    if s["causal"]:
        mask = mask & (j <= t.unsqueeze(1) + (klens - qlens).unsqueeze(2))
    mask = mask.unsqueeze(1)
    S = (q @ k.transpose(2, 3).contiguous()) * scale
    top = S.masked_fill(~mask, -math.inf).amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    P = torch.exp((S - top).masked_fill(~mask, -math.inf))
    total = P.sum(dim=3, keepdim=True)
    P = P / torch.where(total == 0, 1.0, total)
    O = P @ v
    qrows, krows = s["q"].shape[0], s["k"].shape[0]
    out = _plain_scatter(O, qat, qlive, qrows, torch.bfloat16)
    if s["dO"] is None:
        return out
    lse = torch.full((H, qrows + 1), -math.inf, device="cuda")
    lse[:, torch.where(qlive, qat, qrows)] = (top + torch.log(total)).squeeze(3).transpose(0, 1)
    dO = _plain_gather(s["dO"], H, qat, qlive)
    dP = dO @ v.transpose(2, 3).contiguous()
    dS = P * (dP - (dO * O).sum(dim=3, keepdim=True)) * scale
    heads = lambda x: x.unflatten(1, (Hk, -1)).sum(dim=2)
    dq = dS @ k
    dk, dv = heads(dS.transpose(2, 3).contiguous() @ q), heads(P.transpose(2, 3).contiguous() @ dO)
    return [out, lse[:, :qrows].contiguous(), _plain_scatter(dq, qat, qlive, qrows, torch.bfloat16),
            _plain_scatter(dk, kat, klive, krows, torch.bfloat16),
            _plain_scatter(dv, kat, klive, krows, torch.bfloat16)]


# ---- the library's calls ----------------------------------------------------

def _own_norm(s):
    from paper_2607_08526_amd import qlinear as ql
    if s["y"] != "int8":
        return ql.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], ydtype=_dtype(s["y"]))
    qx, sx, h = ql.rms_norm_int8(s["x"], s["weight"], EPS, residual=s["residual"])
    values = torch.empty(qx.shape, dtype=torch.bfloat16, device=qx.device)
    return torch.mul(qx, sx.view(torch.float16).float().unsqueeze(1), out=values), h


def _own_norm_grad(s):
    from paper_2607_08526_amd import qlinear as ql
    return ql.rms_norm_backward(s["dy"], s["h"], s["weight"], EPS, dres=s["dres"],
                                dtype=s["dres"].dtype, weight_grad=s["weight"] is not None)


def _own_attend(s):
    from paper_2607_08526_amd import qlinear as ql
    shape = (s["B"], s["T"], s["H"])
    how = dict(kv_heads=s["Hk"], dh=s["dh"], kT=s["kT"], causal=s["causal"],
               q_offsets=s["q_offsets"], k_offsets=s["k_offsets"], q_lens=s["q_lens"],
               k_lens=s["k_lens"])
    if s["dO"] is None:
        return ql.attention_forward(s["q"], s["k"], s["v"], *shape, **how, with_lse=False)[0]
    O, lse = ql.attention_forward(s["q"], s["k"], s["v"], *shape, **how)
    g = ql.attention_backward(s["q"], s["k"], s["v"], O, lse, s["dO"], *shape, **how)
    return [O, lse, g.q, g.k, g.v]


# ---- prepare and run -------------------------------------------------------

def prepare(case, seed):
    kind = case["kind"]
    if kind == "norm":
        x, residual, weight = _norm_inputs(case, seed)
        return {"kind": kind, "x": x, "residual": residual, "weight": weight, "y": case["y"]}
    if kind == "norm_grad":
        dy, h, weight, dres = _norm_inputs(case, seed)
        return {"kind": kind, "dy": dy, "h": h, "weight": weight, "dres": dres}
    q, k, v, dO, qside, kside = _attend_inputs(case, seed)
    state = {**case, "q": q, "k": k, "v": v, "dO": dO}
    for side, (first, lens), rows in (("q", qside, q.shape[0]), ("k", kside, k.shape[0])):
        i64 = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
        own_rows = case["rows"] if side == "k" or case["T"] == case["kT"] else "full"
        state[side + "first"], state[side + "lens"] = i64(first), i64(lens)
        state[side + "_offsets"] = i64(first + [first[-1] + lens[-1]]) if own_rows == "packed" \
            else None
        state[side + "_lens"] = state[side + "lens"] if own_rows == "padded" else None
    return state


def run(state):
    form = {"norm": (_plain_norm, _own_norm), "norm_grad": (_plain_norm_grad, _own_norm_grad),
            "attend": (_plain_attend, _own_attend), "train": (_plain_attend, _own_attend)}
    return form[state["kind"]][1 if own else 0](state)


def work(case):
    size = {"f32": 4, "bf16": 2, "int8": 1}
    if case["kind"] in ("norm", "norm_grad"):
        M, N = case["M"], case["N"]
        weight = 4 * N if case["w"] else 0
        if case["kind"] == "norm":
            return {"bytes": M * N * (size[case["x"]] + 2 * size[case["h"]] + size[case["y"]])
                    + weight + (2 * M if case["y"] == "int8" else 0), "flops": 5 * M * N}
        return {"bytes": M * N * (size[case["x"]] + size[case["h"]] + 2 * size[case["dx"]])
                + 2 * weight, "flops": 12 * M * N}
    order = list(range(case["B"]))
    (_, _, qlens), (_, _, klens) = (_rows(case, s, order) for s in (0, 1))
    pairs = 0
    for a, b in zip(qlens, klens):
        # causal: query i sees i + b - a + 1 keys, none where that is negative
        pairs += sum(max(0, i + b - a + 1) for i in range(a)) if case["causal"] else a * b
    wide, narrow, train = case["H"] * case["dh"], case["Hk"] * case["dh"], case["kind"] == "train"
    # train: q, o, dO, dq, and k, v, dk, dv, and the row sums' logarithms
    return {"bytes": 2 * ((4 if train else 2) * sum(qlens) * wide
                          + (4 if train else 2) * sum(klens) * narrow)
            + (4 * case["H"] * sum(qlens) if train else 0),
            "flops": (14 if train else 4) * case["dh"] * case["H"] * pairs}


# ---- the operators in 64 bits ------------------------------------------------

def _exact_unit(v):
    return v / torch.sqrt(torch.linalg.vector_norm(v, dim=1, keepdim=True) ** 2 / v.shape[1] + EPS)


def exact(case, seed):
    if case["kind"] == "norm":
        x, residual, weight = _norm_inputs(case, seed)
        h = x.double() + residual.double()
        if case["y"] == "int8":  # the codes are those of the fp32 sum
            y = _exact_unit((x.float() + residual.float()).double())
        else:
            y = _exact_unit(h)
        if weight is not None:
            y = y * weight.double()
        if case["y"] == "int8":
            y = y.float().double()
            scale = (y.abs().max(dim=1, keepdim=True).values / 127).half().double()
            y = torch.round(y / scale).clamp(-127, 127) * scale
        return y, h
    if case["kind"] == "norm_grad":
        dy, h, weight, dres = _norm_inputs(case, seed)
        h = h.double().requires_grad_()
        w = (torch.ones(case["N"], device="cuda") if weight is None else weight).double()
        w.requires_grad_()
        dh, dw = torch.autograd.grad(_exact_unit(h) * w, (h, w), dy.double())
        return dh + dres.double(), None if weight is None else dw
    q, k, v, dO, (qfirst, qlens), (kfirst, klens) = _attend_inputs(case, seed)
    H, Hk, dh = case["H"], case["Hk"], case["dh"]
    out = [torch.zeros_like(x, dtype=torch.float64) for x in (q, q, k, v)]
    lse = torch.full((H, q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    for a, n, b, m in zip(qfirst, qlens, kfirst, klens):
        skip = max(0, n - m) if case["causal"] else 0  # queries that see no key
        a, n = a + skip, n - skip
        split = lambda x, at, len_: x[at: at + len_].double().reshape(len_, -1, dh).permute(1, 0, 2)
        leaves = [split(*t).contiguous().requires_grad_(dO is not None)
                  for t in ((q, a, n), (k, b, m), (v, b, m))]
        Q, K, V = leaves
        K, V = (x[:, None].expand(Hk, H // Hk, m, dh).reshape(H, m, dh) for x in (K, V))
        S = torch.matmul(Q, K.permute(0, 2, 1).contiguous()) / math.sqrt(dh)
        if case["causal"]:
            later = torch.ones(n, m, dtype=torch.bool, device="cuda").triu(m - n + 1)
            S = torch.where(later, -math.inf, S)
        L = torch.logsumexp(S, dim=2)
        O = torch.matmul(torch.exp(S - L.unsqueeze(2)), V)
        join = lambda x: x.detach().permute(1, 0, 2).reshape(x.shape[1], -1)
        out[0][a: a + n] = join(O)
        lse[:, a: a + n] = L.detach()
        if dO is not None:
            grads = torch.autograd.grad(O, leaves, split(dO, a, n).contiguous())
            for to, at, g in ((out[1], a, grads[0]), (out[2], b, grads[1]), (out[3], b, grads[2])):
                to[at: at + g.shape[1]] = join(g)
    return out[0] if dO is None else [out[0], lse, *out[1:]]
