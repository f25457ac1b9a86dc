"""The masked attention and its backward pass on the GPU against 64-bit references
(train_ref.py derives the tolerances)."""
import math

import numpy as np
import pytest

import train_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def host(t):
    return t.double().cpu().numpy()


def i64(torch, x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


class Case:
    """Random rows and where the sequences lie in them.  Rows that are padding or of no
    sequence hold NaN and infinities.  lens, klens: of the sequences (None: full)."""

    def __init__(self, torch, B, T, H, Hk=None, dh=64, kT=None, causal=False, rows="full",
                 lens=None, klens=None, size=1.0, seed=0, pad=0, scale=None):
        kT, Hk = T if kT is None else kT, H if Hk is None else Hk
        rng = np.random.default_rng(seed + 1000 * T + kT + 7 * H + dh)
        klens = lens if klens is None and T == kT else klens
        qlens = [T] * B if lens is None else lens
        kl = [kT] * B if klens is None else klens
        self.how = dict(kv_heads=Hk, dh=dh, kT=kT, causal=causal, scale=scale)
        self.shape = (B, T, H)
        place = {}
        for side, given, ls, most in (("q", lens, qlens, T), ("k", klens, kl, kT)):
            off = lens_ = None
            if rows == "packed" and given is not None:
                first = [3 + sum(ls[:b]) for b in range(B)]  # rows 0 to 2 are of none
                off = i64(torch, first + [3 + sum(ls)])
                total, caps = 3 + sum(ls) + 5, ls
            elif rows == "both" and given is not None:
                caps = [x + 2 * (b % 3) for b, x in enumerate(ls)]
                first = [sum(caps[:b]) for b in range(B)]
                off, lens_ = i64(torch, first + [sum(caps)]), i64(torch, ls)
                caps = [min(c, most) for c in caps]
                total = first[-1] + caps[-1] + 9
            else:
                first, caps, total = [b * most for b in range(B)], [most] * B, B * most
                lens_ = i64(torch, ls) if given is not None else None
            self.how[side + "_offsets"], self.how[side + "_lens"] = off, lens_
            place[side] = (list(zip(first, ls, caps)), total)
        self.seqs = [R.Seq(a, b) for a, b in zip(place["q"][0], place["k"][0])]

        def make(side, heads, std):
            places, total = place[side]
            x = np.full((total, heads * dh + pad), np.nan, np.float32)
            x[::2] = np.inf
            for first, n, _ in places:
                x[first: first + n] = rng.standard_normal((n, heads * dh + pad)) * std
            t = torch.from_numpy(x).to(torch.bfloat16).cuda()
            return t[:, : heads * dh]

        self.q, self.k, self.v = make("q", H, size), make("k", Hk, 1.0), make("k", Hk, 1.0)
        self.dO = make("q", H, 0.1)
        self.scale = 1 / math.sqrt(dh) if scale is None else scale

    def want(self, out_bf16=True, grads=False, grad_bf16=True):
        B, T, H = self.shape
        return R.attention(*(host(t) for t in (self.q, self.k, self.v)), self.seqs, H,
                           self.how["kv_heads"], self.how["dh"], self.scale, self.how["causal"],
                           out_bf16, host(self.dO) if grads else None, grad_bf16)


def compare(got, want, name):
    value, bound = want[name]
    of = ~np.isnan(value)  # rows of sequences
    got = host(got)
    with np.errstate(invalid="ignore"):
        bad = of & ~((np.abs(got - value) <= bound) | (got == value))
    assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], value[bad][:4], bound[bad][:4])
    return of, got


def check_forward(torch, ql, c, odtype=None):
    odtype = odtype or torch.bfloat16
    O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, odtype=odtype, **c.how)
    want = c.want(odtype == torch.bfloat16)
    of, got = compare(O, want, "O")
    assert (got[~of] == 0).all()
    of, got = compare(lse, want, "lse")
    assert (got[~of] == -np.inf).all()
    return O, lse


# one key and query, tiles' ends, odd, few and many keys, each side longer; every
# kernel: one to four key groups, split keys, both head sizes
FORWARD = [
    dict(B=1, T=1, H=1), dict(B=2, T=1, H=3, kT=77), dict(B=1, T=1, H=8, Hk=1, kT=5000),
    dict(B=3, T=1, H=16, Hk=4, kT=1500), dict(B=1, T=3, H=4, Hk=2, kT=700),
    dict(B=1, T=31, H=1, kT=33), dict(B=1, T=33, H=1, kT=31), dict(B=2, T=64, H=2),
    dict(B=1, T=65, H=2, kT=63), dict(B=1, T=107, H=6, Hk=2), dict(B=2, T=130, H=2, kT=257),
    dict(B=4, T=640, H=8), dict(B=1, T=1200, H=2), dict(B=2, T=300, H=32),
    dict(B=1, T=129, H=5, kT=1), dict(B=1, T=200, H=1, kT=4000), dict(B=3, T=33, H=40, kT=130),
    dict(B=1, T=1, H=1, kT=344),
]
# (parts of the keys where no wavefronts share them, D = 64)
LARGE = dict(B=3, T=23, H=27, Hk=9, kT=10300)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", FORWARD, ids=lambda s: "-".join(map(str, s.values())))
def test_forward(gpu, shape, causal, dh):
    torch, ql = gpu
    check_forward(torch, ql, Case(torch, **shape, causal=causal, dh=dh, size=2.0, pad=8))


LENGTHS = [
    dict(B=4, T=100, H=2, lens=[100, 1, 0, 37]),
    dict(B=3, T=300, H=4, Hk=2, lens=[299, 65, 128]),
    dict(B=3, T=40, H=2, lens=[40, 7, 0], kT=90, klens=[0, 5, 90]),
    dict(B=2, T=1, H=8, Hk=2, kT=900, klens=[900, 13]),
    dict(B=5, T=2, H=8, Hk=1, kT=700, klens=[1, 0, 699, 64, 2]),
    dict(B=2, T=700, H=2, lens=[513, 700]),
    dict(B=1, T=150, H=1, lens=[77], kT=40, klens=[33]),
]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("rows", ["padded", "packed", "both"])
@pytest.mark.parametrize("shape", LENGTHS, ids=lambda s: "-".join(map(str, s.values())))
def test_forward_lengths(gpu, shape, rows, causal, dh):
    """Sequences of unlike lengths, with empty ones and queries that see no key; what
    padding rows hold does not matter."""
    torch, ql = gpu
    check_forward(torch, ql, Case(torch, **shape, rows=rows, causal=causal, dh=dh))


def test_forward_large(gpu):
    torch, ql = gpu
    check_forward(torch, ql, Case(torch, **LARGE, rows="padded", klens=[10300, 1, 7777]))


def test_forward_types_and_scales(gpu):
    torch, ql = gpu
    check_forward(torch, ql, Case(torch, 2, 150, 3), torch.float32)
    check_forward(torch, ql, Case(torch, 1, 1, 4, Hk=1, kT=3000), torch.float32)
    check_forward(torch, ql, Case(torch, 2, 90, 2, scale=0.0, causal=True))
    # scores up to several hundred: a row's probability is nearly one key's
    for dh in (64, 128):
        check_forward(torch, ql, Case(torch, 1, 200, 2, dh=dh, size=60.0, causal=True))
        check_forward(torch, ql, Case(torch, 1, 2, 4, Hk=2, dh=dh, kT=2000, size=60.0))


def test_forward_rising_scores(gpu):
    """Every tile's scores far above the one before: the maximum moves each time."""
    torch, ql = gpu
    for dh in (64, 128):
        c = Case(torch, 1, 70, 2, dh=dh, kT=600)
        ramp = torch.linspace(0, 6, 600, device="cuda").unsqueeze(1)
        c.q[:] = c.q.abs() + 0.5
        c.k[:] = (c.k.float() * 0.1 + ramp).to(torch.bfloat16)
        check_forward(torch, ql, c)


def test_forward_keeps_other_rows(gpu):
    """Rows of no sequence keep what they held, columns behind the heads too."""
    torch, ql = gpu
    for split in (False, True):
        c = Case(torch, 3, 1 if split else 90, 2, kT=900 if split else 90, rows="packed",
                 lens=[1, 0, 1] if split else [90, 11, 4], klens=[900, 5, 65] if split else None)
        rows = c.q.shape[0]
        O = torch.full((rows, 128 + 4), 7.0, device="cuda", dtype=torch.bfloat16)
        lse = torch.full((2, rows), 7.0, device="cuda")
        got, sums = ql.attention_forward(c.q, c.k, c.v, *c.shape, O=O[:, :128], lse=lse, **c.how)
        assert got.data_ptr() == O.data_ptr() and sums is lse
        want = c.want()
        of, g = compare(got, want, "O")
        assert (g[~of] == 7).all() and (O[:, 128:] == 7).all()
        of, g = compare(lse, want, "lse")
        assert (g[~of] == 7).all()
        # (offsets that fall or leave the tensor: every access stays inside of it)
        for bad in ([0, 10 ** 12, -5, 2], [rows, 0, rows, rows], [-7, -3, -1, -1]):
            how = c.how | dict(q_offsets=i64(torch, bad))
            ql.attention_forward(c.q, c.k, c.v, *c.shape, O=O[:, :128], lse=lse, **how)
        torch.cuda.synchronize()


def test_forward_equals_itself(gpu):
    """Bit for bit again, and each sequence as it is alone."""
    torch, ql = gpu
    c = Case(torch, 3, 200, 4, Hk=2, rows="packed", lens=[200, 50, 131], causal=True)
    O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
    for _ in range(3):
        again = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
        assert torch.equal(O, again[0]) and torch.equal(lse, again[1])
    assert ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how, with_lse=False)[1] is None


def test_forward_as_attention(gpu):
    """Against the unmasked entry point where both apply (each is off by its bound)."""
    torch, ql = gpu
    c = Case(torch, 2, 333, 4)
    O, _ = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
    plain = ql.attention(c.q.contiguous(), c.k.contiguous(), c.v.contiguous(), *c.shape,
                         odtype=torch.bfloat16)
    bound = c.want()["O"][1]
    assert (np.abs(host(O) - host(plain)) <= 2 * bound).all()


def check_backward(torch, ql, c, dtype=None, odtype=None):
    dtype, odtype = dtype or torch.bfloat16, odtype or torch.bfloat16
    O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, odtype=odtype, **c.how)
    g = ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, dtype=dtype, **c.how)
    want = c.want(odtype == torch.bfloat16, True, dtype == torch.bfloat16)
    for name, t in (("dv", g.v), ("dk", g.k), ("dq", g.q)):
        assert t.dtype == dtype
        of, got = compare(t, want, name)
        assert (got[~of] == 0).all()
    return O, lse, g


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [s for s in FORWARD if s["B"] * s["T"] * s["H"] < 9000],
                         ids=lambda s: "-".join(map(str, s.values())))
def test_backward(gpu, shape, causal, dh):
    torch, ql = gpu
    check_backward(torch, ql, Case(torch, **shape, causal=causal, dh=dh, size=2.0, pad=8))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("rows", ["padded", "packed", "both"])
@pytest.mark.parametrize("shape", LENGTHS, ids=lambda s: "-".join(map(str, s.values())))
def test_backward_lengths(gpu, shape, rows, causal, dh):
    torch, ql = gpu
    check_backward(torch, ql, Case(torch, **shape, rows=rows, causal=causal, dh=dh))


def test_backward_types_and_scales(gpu):
    torch, ql = gpu
    check_backward(torch, ql, Case(torch, 2, 150, 3), torch.float32)
    check_backward(torch, ql, Case(torch, 2, 150, 4, Hk=2, dh=128), torch.float32, torch.float32)
    check_backward(torch, ql, Case(torch, 2, 90, 2, scale=0.0, causal=True))
    for dh in (64, 128):
        check_backward(torch, ql, Case(torch, 1, 200, 2, dh=dh, size=30.0, causal=True))
    # parts of the reductions: keys for a few queries, queries (of several heads) for few keys
    check_backward(torch, ql, Case(torch, 1, 5, 2, kT=3000))
    check_backward(torch, ql, Case(torch, 1, 700, 8, Hk=1, dh=128, causal=True), torch.float32)


def test_backward_against_differences(gpu):
    """Central differences of the 64-bit forward's <O, dO> along random directions of
    q, k and v, with steps of 1e-4; their own error, 1e-8 / 6 of a third derivative, is
    below a thousandth of the bound's sum (scores move by |direction| sqrt(dh) * 1e-4)."""
    torch, ql = gpu
    c = Case(torch, 1, 48, 2, Hk=1, kT=60, causal=True)
    _, _, g = check_backward(torch, ql, c, torch.float32)
    want = c.want(True, True, False)
    args = lambda x: (*x, c.seqs, 2, 1, 64, c.scale, True, True)
    base = [host(t) for t in (c.q, c.k, c.v)]
    dO = host(c.dO)
    rng = np.random.default_rng(5)
    for i, (name, got) in enumerate((("dq", g.q), ("dk", g.k), ("dv", g.v))):
        for _ in range(3):
            d = rng.standard_normal(base[i].shape)
            value = []
            for t in (1e-4, -1e-4):
                x = list(base)
                x[i] = base[i] + t * d
                value.append((R.attention(*args(x))["O"][0] * dO).sum())
            diff = (value[0] - value[1]) / 2e-4
            bound = (want[name][1] * np.abs(d)).sum()
            assert abs((host(got) * d).sum() - diff) <= 1.001 * bound


def test_backward_keeps_other_rows(gpu):
    """Gradients as the columns of a fused QKV gradient: rows of no sequence and the
    columns behind keep what they held; only dq on request."""
    torch, ql = gpu
    c = Case(torch, 3, 90, 4, Hk=2, rows="packed", lens=[90, 11, 4], causal=True)
    rows = c.q.shape[0]
    O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
    for dtype in (torch.bfloat16, torch.float32):
        d = torch.full((rows, 512 + 8), 7.0, device="cuda", dtype=dtype)
        dq, dk, dv = d[:, :256], d[:, 256:384], d[:, 384:512]
        g = ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, dq=dq, dk=dk, dv=dv,
                                  **c.how)
        assert g.q is dq and g.k is dk and g.v is dv
        want = c.want(True, True, dtype == torch.bfloat16)
        for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
            of, got = compare(t, want, name)
            assert (got[~of] == 7).all()
        assert (d[:, 512:] == 7).all()
        only = ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, kv_grads=False,
                                     dtype=dtype, **c.how)
        live = torch.from_numpy(~np.isnan(want["dq"][0])).cuda()
        assert only.k is None and only.v is None and torch.equal(only.q[live], dq[live])
    for bad in ([0, 10 ** 12, -5, 2], [rows, 0, rows, rows]):
        how = c.how | dict(q_offsets=i64(torch, bad), k_offsets=i64(torch, bad))
        ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, **how)
    torch.cuda.synchronize()


def test_backward_equals_itself(gpu):
    """Bit for bit the same again (no sum's order depends on anything but the sizes)."""
    torch, ql = gpu
    for c in (Case(torch, 2, 300, 8, Hk=2, causal=True), Case(torch, 1, 700, 4, Hk=1, dh=128)):
        O, lse, g = check_backward(torch, ql, c)
        for _ in range(4):
            again = ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, **c.how)
            assert all(torch.equal(a, b) for a, b in zip(g, again))


def test_no_rows(gpu):
    """No sequences, no queries, no keys: zeros where there are rows, and no fault."""
    torch, ql = gpu
    q, none = torch.randn((6, 128), device="cuda").to(torch.bfloat16), None
    none = q[:0]
    O, lse = ql.attention_forward(q, none, none, 2, 3, 2, kT=0)
    assert (O == 0).all() and (lse == -math.inf).all()
    g = ql.attention_backward(q, none, none, O, lse, q, 2, 3, 2, kT=0)
    assert (g.q == 0).all() and g.k.shape == (0, 128)
    O, lse = ql.attention_forward(none, q, q, 2, 0, 2, kT=3)
    assert O.shape == (0, 128) and lse.shape == (2, 0)
    g = ql.attention_backward(none, q, q, O, lse, none, 2, 0, 2, kT=3)
    assert (g.k == 0).all() and (g.v == 0).all()
    O, lse = ql.attention_forward(q, q, q, 0, 3, 2)
    assert (O == 0).all() and (lse == -math.inf).all()


def test_graph(gpu):
    """Forward and backward captured, replayed on other inputs and lengths between eager
    calls (split reductions and their joins among them)."""
    torch, ql = gpu
    for c in (Case(torch, 2, 130, 4, Hk=2, rows="padded", lens=[130, 60], causal=True),
              Case(torch, 1, 2, 4, Hk=1, dh=128, kT=2000)):
        def step():
            O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
            return (O, lse, *ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, **c.how))

        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            step()
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
        for k in range(4):
            for t in (c.q, c.k, c.v, c.dO):
                t.normal_()
            if c.how["k_lens"] is not None:
                for name in ("q_lens", "k_lens"):
                    c.how[name].copy_(i64(torch, [130 - 40 * k, 7 + k]))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            copies = [t.clone() for t in got]
            for a, b in zip(copies, step()):
                assert torch.equal(a, b)
            torch.cuda.synchronize()
