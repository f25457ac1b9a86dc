"""The operators of include/qlinear_train.h where calls meet each other, the library's
other operators, or the ends of their ranges: a block forward and backward, threads on
one stream, graphs that share a workspace, outputs made on another stream, rows far
apart."""
import threading

import numpy as np
import pytest

import block_ref as BR
import train_ref as R
from test_gpu_norm import host, within
from test_gpu_train_attention import Case, check_backward, check_forward, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


class Block:
    """A transformer block on frozen MXFP4 weights, forward and backward, of two packed
    sequences: norm, QKV with rotary positions, causal attention with shared key heads,
    the residual's addition in the next norm, the gated pair, down."""

    H, HK, DH, HIDDEN, EPS = 4, 2, 64, 512, 1e-6
    LENS = [70, 41]

    def __init__(self, torch, ql, seed=0):
        self.torch, self.ql = torch, ql
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        new = lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda") * std
        self.d, self.wide = self.H * self.DH, (self.H + 2 * self.HK) * self.DH
        rows = self.rows = sum(self.LENS)
        self.weights = {}
        for name, n, k in (("qkv", self.wide, self.d), ("out", self.d, self.d),
                           ("gate", self.HIDDEN, self.d), ("up", self.HIDDEN, self.d),
                           ("down", self.d, self.HIDDEN)):
            w = ql.quantize(ql.FMT_MXFP4, new(n, k, std=k ** -0.5))
            self.weights[name] = (w, ql.dequantize(ql.FMT_MXFP4, *w))
        self.n1, self.n2 = (1 + new(self.d, std=0.2) for _ in range(2))
        self.x, self.dy = new(rows, self.d), new(rows, self.d, std=0.1)
        i64 = lambda v: torch.tensor(v, dtype=torch.int64, device="cuda")
        self.offsets = i64([0, self.LENS[0], rows])
        self.positions = torch.cat([torch.arange(n, device="cuda") for n in self.LENS])
        self.freqs, _ = ql.rotary_frequencies(self.DH)
        self.how = dict(kv_heads=self.HK, dh=self.DH, causal=True, q_offsets=self.offsets,
                        k_offsets=self.offsets)
        self.seqs = [R.Seq((a, n, n), (a, n, n)) for a, n in ((0, self.LENS[0]),
                                                             (self.LENS[0], self.LENS[1]))]

    def linear(self, name, x, dtype):
        (codes, scales), w = self.weights[name]
        return self.ql.forward_ep(self.ql.FMT_MXFP4, x, codes, scales, w.shape[0], ydtype=dtype)

    def split(self, qkv):
        return qkv.split([self.d, self.HK * self.DH, self.HK * self.DH], dim=1)

    def forward(self):
        ql, bf = self.ql, self.torch.bfloat16
        s = self.s = {}
        s["a"], _ = ql.rms_norm(self.x, self.n1, self.EPS)
        s["qkv"] = self.linear("qkv", s["a"], bf)
        s["raw"] = s["qkv"].clone()
        ql.rotary(s["qkv"][:, : (self.H + self.HK) * self.DH], self.H + self.HK, self.freqs,
                  dh=self.DH, positions=self.positions)
        q, k, v = self.split(s["qkv"])
        s["O"], s["lse"] = ql.attention_forward(q, k, v, 2, max(self.LENS), self.H, **self.how)
        s["o"] = self.linear("out", s["O"], self.torch.float32)
        s["b"], s["h"] = ql.rms_norm(s["o"], self.n2, self.EPS, residual=self.x)
        s["H"] = ql.gated_forward(ql.FMT_MXFP4, s["b"], self.weights["gate"][0],
                                  self.weights["up"][0])
        return s["h"] + self.linear("down", s["H"], self.torch.float32)

    def backward(self):
        """The gradients of x, of both norms' weights, from dy."""
        ql, bf, s = self.ql, self.torch.bfloat16, self.s
        dH = (self.dy @ self.weights["down"][1]).to(bf)
        s["db"] = ql.gated_backward(ql.FMT_MXFP4, s["b"], self.weights["gate"][0],
                                    self.weights["up"][0], dH).X
        s["dh"], s["dn2"] = ql.rms_norm_backward(s["db"], s["h"], self.n2, self.EPS, dres=self.dy)
        s["dO"] = (s["dh"] @ self.weights["out"][1]).to(bf)
        s["dqkv"] = self.torch.empty_like(s["qkv"])
        q, k, v = self.split(s["qkv"])
        dq, dk, dv = self.split(s["dqkv"])
        ql.attention_backward(q, k, v, s["O"], s["lse"], s["dO"], 2, max(self.LENS), self.H,
                              dq=dq, dk=dk, dv=dv, **self.how)
        s["grads"] = [t.clone() for t in (dq, dk, dv)]
        ql.rotary(s["dqkv"][:, : (self.H + self.HK) * self.DH], self.H + self.HK, self.freqs,
                  dh=self.DH, positions=self.positions, adjoint=True)
        s["da"] = s["dqkv"].float() @ self.weights["qkv"][1]
        s["dx"], s["dn1"] = ql.rms_norm_backward(s["da"], self.x, self.n1, self.EPS, dres=s["dh"])
        return s["dx"], s["dn1"], s["dn2"]

    def exact(self):
        """The same in 64 bits by torch's own differentiation, with no rounding between."""
        torch = self.torch
        w = {n: v[1].double() for n, v in self.weights.items()}
        leaves = [t.double().requires_grad_() for t in (self.x, self.n1, self.n2)]
        x, n1, n2 = leaves
        norm = lambda v, n: v * n / torch.sqrt((v * v).mean(dim=1, keepdim=True) + self.EPS)
        qkv = norm(x, n1) @ w["qkv"].T
        t = self.positions.double()[:, None] * self.freqs
        c, sn = torch.cos(t)[:, None, :], torch.sin(t)[:, None, :]
        both = qkv[:, : (self.H + self.HK) * self.DH].reshape(self.rows, -1, self.DH)
        a, b = both.chunk(2, dim=2)
        both = torch.cat((a * c - b * sn, b * c + a * sn), dim=2)
        q, k = both[:, : self.H], both[:, self.H:].repeat_interleave(self.H // self.HK, dim=1)
        v = qkv[:, (self.H + self.HK) * self.DH:].reshape(self.rows, self.HK, self.DH)
        v = v.repeat_interleave(self.H // self.HK, dim=1)
        at = torch.arange(self.rows, device="cuda")
        seq = (at >= self.LENS[0]).long()
        see = (seq[:, None] == seq) & (at <= at[:, None])
        S = torch.stack([q[:, h] @ k[:, h].T for h in range(self.H)]) * self.DH ** -0.5
        P = torch.softmax(torch.where(see, S, -torch.inf), dim=2)
        o = torch.cat([P[h] @ v[:, h] for h in range(self.H)], dim=1)
        h = x + o @ w["out"].T
        z = norm(h, n2)
        g = z @ w["gate"].T
        y = h + (g * torch.sigmoid(g) * (z @ w["up"].T)) @ w["down"].T
        return y.detach(), torch.autograd.grad(y, leaves, self.dy.double())


def test_block(gpu):
    """Each of the new stages against 64 bits on its own inputs, element by element; then
    the block's output and gradients against the 64-bit composition.  Between the two lie
    nine values that are rounded to bf16 forward (a, qkv, rotated, P, O, b, G U of the pair
    and H) and as many backward; each is off by at most 2^-8 of its size and at random, so
    the norm of the whole, if every rounding passed on in full, is off by less than
    sqrt(18) 2^-8 = 0.017; held below 0.02 (products between stages have gains below 1
    and above, which this does not count: it is a check of the composition, the bounds
    are the stages')."""
    torch, ql = gpu
    b = Block(torch, ql)
    y = b.forward()
    dx, dn1, dn2 = b.backward()
    s = b.s
    H, HK, DH = b.H, b.HK, b.DH
    want = R.norm(host(b.x), host(b.n1), b.EPS)
    within(host(s["a"]), want, R.norm_error(want, True))
    assert torch.equal(s["h"], s["o"] + b.x)
    want = R.norm(host(s["h"]), host(b.n2), b.EPS)
    within(host(s["b"]), want, R.norm_error(want, True))
    turned = (H + HK) * DH
    raw = host(s["raw"])
    want, err = BR.rotary(raw[:, :turned], H + HK, DH, host(b.freqs), b.positions.cpu().numpy(),
                          False, 1.0, False)
    within(host(s["qkv"][:, :turned]), want, err + R.BF16 * (np.abs(want) + err))
    q, k, v = (host(t) for t in b.split(s["qkv"]))
    want = R.attention(q, k, v, b.seqs, H, HK, DH, DH ** -0.5, True, True, host(s["dO"]), True)
    for name, t in zip(("O", "lse", "dq", "dk", "dv"), (s["O"], s["lse"], *s["grads"])):
        assert compare(t, want, name)[0].all()
    for d, h, w, res, got, gw in (("db", s["h"], b.n2, b.dy, s["dh"], dn2),
                                  ("da", b.x, b.n1, s["dh"], dx, dn1)):
        wx, ww, ex, ew = R.norm_grads(host(s[d]), host(h), host(w), b.EPS, host(res))
        within(host(got), wx, ex)
        within(host(gw), ww, ew)
    ey, grads = b.exact()
    off = lambda t, e: float((t.double() - e).norm() / e.norm())
    errors = [off(t, e) for t, e in zip((y, dx, dn1, dn2), (ey, *grads))]
    assert max(errors) < 0.02, errors


def test_block_graph(gpu):
    """The block forward and backward captured whole, replayed on other inputs with eager
    calls of the same between, bit for bit."""
    torch, ql = gpu
    b = Block(torch, ql, 1)
    step = lambda: (b.forward(), *b.backward())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = step()
    for _ in range(3):
        b.x.normal_()
        b.dy.normal_(std=0.1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        copies = [t.clone() for t in got]
        for a, c in zip(copies, step()):
            assert torch.equal(a, c)
        torch.cuda.synchronize()


def calls(torch, ql):
    """Calls that use a workspace, each with its result."""
    few = Case(torch, 2, 1, 8, Hk=2, kT=3000)
    many = Case(torch, 1, 500, 8, Hk=1, dh=128, causal=True)
    x, w = torch.randn((700, 900), device="cuda"), torch.rand(900, device="cuda")
    back = {}
    for name, c in (("few", few), ("many", many)):
        back[name] = (c, *ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how))
    return [lambda: ql.attention_forward(few.q, few.k, few.v, *few.shape, **few.how),
            lambda: ql.attention_backward(many.q, many.k, many.v, *back["many"][1:], many.dO,
                                          *many.shape, **many.how),
            lambda: ql.attention_backward(few.q, few.k, few.v, *back["few"][1:], few.dO,
                                          *few.shape, **few.how),
            lambda: ql.rms_norm_backward(x, x, w)]


def test_threads_on_one_stream(gpu):
    torch, ql = gpu
    work = calls(torch, ql)
    want = [[t.clone() for t in c()] for c in work]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    fails = []

    def run(k):
        with torch.cuda.stream(stream):
            for _ in range(40):
                got = work[k]()
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[k])):
                    fails.append(k)

    threads = [threading.Thread(target=run, args=(k,)) for k in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not fails


def test_graphs_share_a_workspace(gpu):
    """Two graphs captured on one stream, replayed in turn with eager calls between."""
    torch, ql = gpu
    work = calls(torch, ql)
    want = [[t.clone() for t in c()] for c in work]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for c in work:
            c()
    torch.cuda.synchronize()
    graphs = []
    for half in (work[:2], work[2:]):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = [c() for c in half]
        graphs.append((graph, got))
    for _ in range(4):
        for (graph, got), expected in zip(graphs, (want[:2], want[2:])):
            for r in got:
                for t in r:
                    t.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for r, e in zip(got, expected):
                assert all(torch.equal(a, b) for a, b in zip(r, e))
            with torch.cuda.stream(stream):
                for c, e in zip(work, want):
                    assert all(torch.equal(a, b) for a, b in zip(c(), e))
            torch.cuda.synchronize()


def test_capture_without_a_workspace(gpu):
    """A stream's first call is a captured one: its workspace is of the graph."""
    torch, ql = gpu
    work = calls(torch, ql)
    want = [[t.clone() for t in c()] for c in work]
    for c, e in zip(work, want):
        stream = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            got = c()
        for _ in range(3):
            for t in got:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, e))


def test_outputs_of_another_stream(gpu):
    """Outputs that a call on a given stream makes come from that stream's memory, also
    those filled first."""
    torch, ql = gpu
    x = torch.randn((64, 256), device="cuda")
    c = Case(torch, 2, 50, 2, rows="packed", lens=[50, 21])
    O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
    work = [lambda s: ql.rms_norm(x, residual=x, stream=s),
            lambda s: ql.rms_norm_int8(x, residual=x, stream=s),
            lambda s: ql.rms_norm_backward(x, x, dres=x, stream=s),
            lambda s: ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how, stream=s),
            lambda s: ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, **c.how,
                                            stream=s)]
    side = torch.cuda.Stream()
    for i, call in enumerate(work):
        want = [t.clone() for t in call(None)]
        torch.cuda.synchronize()
        gone = [torch.empty_like(t) for t in want]
        freed = {t.data_ptr() for t in gone}
        del gone
        got = list(call(side))
        side.synchronize()
        for a, b in zip(got, want):
            assert a.data_ptr() not in freed, i
            assert torch.equal(a, b), i


def test_rows_far_apart(gpu):
    """Row strides whose products pass 32 bits: as the same rows side by side."""
    torch, ql = gpu
    ld, rows = (1 << 24) - 8, 300  # 10 GB
    far = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").as_strided((rows, 1024),
                                                                                (ld, 1))
    far.normal_()
    near = far.contiguous()
    cut = lambda t, a, n: t[:, a: a + n]
    shape = lambda t: (cut(t, 0, 256), cut(t, 256, 128), cut(t, 384, 128))
    for T, kT, dh in ((rows, rows, 64), (2, rows, 128)):
        H, Hk = 256 // dh, 128 // dh
        how = dict(kv_heads=Hk, dh=dh, kT=kT, causal=True)
        out = []
        for t in (far, near):
            q, k, v = shape(t)
            q, k, v = q[:T], k[:kT], v[:kT]
            dO = cut(t, 512, 256)[:T]
            O, lse = ql.attention_forward(q, k, v, 1, T, H, **how)
            g = ql.attention_backward(q, k, v, O, lse, dO, 1, T, H, **how)
            out.append((O, lse, *g))
        for a, b in zip(*out):
            assert torch.equal(a, b)
    # outputs there too: over the columns that nothing else has
    grads = [cut(far, 768, 128), cut(far, 896, 64), cut(far, 960, 64)]
    q, k, v = cut(far, 0, 128), cut(far, 256, 64), cut(far, 384, 64)
    O, lse = ql.attention_forward(q, k, v, 1, rows, 2, kv_heads=1)
    want = ql.attention_backward(q, k, v, O, lse, cut(far, 512, 128), 1, rows, 2, kv_heads=1)
    got = ql.attention_backward(q, k, v, O, lse, cut(far, 512, 128), 1, rows, 2, kv_heads=1,
                                dq=grads[0], dk=grads[1], dv=grads[2])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    near = far.contiguous()  # (with those gradients)
    y, h = ql.rms_norm(far, residual=far)
    y2, h2 = ql.rms_norm(near, residual=near)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    dx, dw = ql.rms_norm_backward(far, far, dx=far)
    dx2, dw2 = ql.rms_norm_backward(near, near, dtype=torch.bfloat16)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_long_cache(gpu):
    """A cache whose keys of one head pass 2^31 elements: far keys count as near ones.  Keys
    are zero but for a few, so that every probability is known: exp(s) / (zeros + sum)."""
    torch, ql = gpu
    n, dh = (1 << 24) + 77, 128
    k = torch.zeros((n, dh), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((n, dh), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, dh), dtype=torch.bfloat16, device="cuda")
    q[0, 0] = 16.0
    for i, at in enumerate((0, 1 << 20, n - 1, n - 78)):
        k[at, 0] = 16.0  # a score of 256 / sqrt(128): e^22.6 times the others' weight
        v[at, i] = 1.0
    O, lse = ql.attention_forward(q, k, v, 1, 1, 1, dh=dh, kT=n, odtype=torch.float32)
    s = 256 / 128 ** 0.5
    total = 4 * np.exp(s) + (n - 4)
    want = np.exp(s) / total
    got = host(O)[0]
    # (bf16 probability, the exponential's and the sum's last steps)
    assert (np.abs(got[:4] - want) <= want * (R.BF16 + 1e-5)).all() and (got[4:] == 0).all()
    assert abs(float(lse) - np.log(total)) <= 1e-5


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("rows", ["padded", "packed"])
def test_causal_over_many_heads(gpu, rows, dh):
    """More (sequence, head) pairs than run at once, short and long ones: those of an XCD
    are taken in groups, the last of them smaller."""
    torch, ql = gpu
    lens = [1 + 37 * b % 130 for b in range(25)]
    c = Case(torch, 25, 130, 32, dh=dh, causal=True, rows=rows, lens=lens)
    check_forward(torch, ql, c)
    check_backward(torch, ql, c)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("how", [
    dict(B=1, T=1, H=2, Hk=1), dict(B=2, T=1, H=2, causal=True), dict(B=1, T=300, H=4, kT=1),
    dict(B=3, T=5, H=4, Hk=2, lens=[1, 5, 1], rows="packed"),
    dict(B=2, T=150, H=2, lens=[150, 1], rows="padded", causal=True),
    dict(B=1, T=700, H=8, Hk=1, kT=1, lens=[690], klens=[1], rows="padded"),
], ids=str)
def test_one_key_has_no_gradient(gpu, how, dh):
    """The softmax of one key is 1 for any score: dq and dk are 0, not what rounding leaves."""
    torch, ql = gpu
    c = Case(torch, **how, dh=dh, size=3.0)
    _, _, g = check_backward(torch, ql, c, torch.float32)
    for s in c.seqs:
        n, m = s.n, s.m
        alone = [i for i in range(n) if (i + m - n == 0 if c.how["causal"] else m == 1)]
        assert m > 1 or alone
        assert (host(g.q)[[s.q + i for i in alone]] == 0).all()
        if m == 1:
            assert (host(g.k)[s.k] == 0).all()
            assert (host(g.v)[s.k] != 0).any()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T, kT, G", [(2, 2, 1), (2, 2, 2), (1, 77, 2), (5, 3, 1), (22, 22, 1),
                                      (40, 100, 2), (64, 64, 2), (128, 128, 1), (97, 33, 1),
                                      (128, 1, 1), (1, 128, 1), (2, 2, 4), (5, 50, 7),
                                      (1, 20, 64)])
def test_few_rows_precisely(gpu, T, kT, G, causal, dh):
    """Gradients of few queries and keys, which the outputs' own type rounds but nothing else
    does: P and dS as two bf16 each (2^-16, and the fp32 roundings before them), the scores'
    and dP's sums of dh fp32 terms, lse and d as these leave them."""
    torch, ql = gpu
    c = Case(torch, 1, T, 2 * G, Hk=2, kT=kT, dh=dh, causal=causal)
    O, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
    g = ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, dtype=torch.float32, **c.how)
    q, k, v, dO = (host(t).astype(np.float64) for t in (c.q, c.k, c.v, c.dO))
    u = 2.0 ** -24
    heads = lambda x, h: x[:, h * dh: (h + 1) * dh]
    for hk in range(2):
        dk, dv, ek, ev = (np.zeros((kT, dh)) for _ in range(4))
        K, V = heads(k, hk), heads(v, hk)
        for h in range(hk * G, (hk + 1) * G):
            Q, W = heads(q, h), heads(dO, h)
            S, Sa = c.scale * Q @ K.T, c.scale * abs(Q) @ abs(K).T
            if causal:
                S[np.arange(kT)[None, :] > np.arange(T)[:, None] + kT - T] = -np.inf
            with np.errstate(invalid="ignore"):
                P = np.exp(S - S.max(1, keepdims=True))
                P = np.nan_to_num(P / P.sum(1, keepdims=True))
            dP, dPa = W @ V.T, abs(W) @ abs(V).T
            d, da = (P * dP).sum(1, keepdims=True), (P * dPa).sum(1, keepdims=True)
            dS = P * (dP - d)
            eP = 2 * (dh + 8) * u * Sa.max(1, keepdims=True) + 2.0 ** -20
            eS = abs(dS) * (1.1 * 2.0 ** -16 + eP) + P * ((dh + 8 + kT) * u * (dPa + da) + eP * da)
            eV = P * (1.1 * 2.0 ** -16 + eP)
            want, bound = c.scale * dS @ K, c.scale * (eS + kT * u * abs(dS)) @ abs(K)
            assert (abs(heads(host(g.q), h) - want) <= bound + 1e-37).all()
            dk += c.scale * dS.T @ Q
            ek += c.scale * (eS + 2 * G * T * u * abs(dS)).T @ abs(Q)
            dv += P.T @ W
            ev += (eV + 2 * G * T * u * P).T @ abs(W)
        assert (abs(heads(host(g.k), hk) - dk) <= ek + 1e-37).all()
        assert (abs(heads(host(g.v), hk) - dv) <= ev + 1e-37).all()
