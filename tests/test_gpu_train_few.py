"""Gradients of few queries over many keys, and of few keys under many queries: the roundings
to bf16 do not average out over outputs of few rows, so P and dS enter their products as two
bf16 each there."""
import numpy as np
import pytest

from test_gpu_train_attention import Case, host

pytestmark = pytest.mark.gpu

u = 2.0 ** -24


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def exact(c, T, kT, G, Hk, dh, causal):
    """O, and of each gradient the value and the bound of its error, from an O in fp32:

    P off by eP of itself: the scores' sums of dh terms in both passes, lse's sum of kT, a
    few roundings of the size of score and lse, the exponential's last steps (2^-20).
    dP by its sum of dh terms; d by dO times O's rounding, its own sum, and the rounding of
    three bf16.  dS and P as two bf16: 2^-16.  Sums over n terms: 2 n u."""
    q, k, v, dO = (host(t).astype(np.float64) for t in (c.q, c.k, c.v, c.dO))
    heads = lambda x, h: x[:, h * dh: (h + 1) * dh]
    out = {n: np.zeros(x.shape) for n, x in (("O", q), ("dq", q), ("dk", k), ("dv", v))}
    err = {n: np.zeros(x.shape) for n, x in out.items()}
    for h in range(Hk * G):
        Q, W, K, V = heads(q, h), heads(dO, h), heads(k, h // G), heads(v, h // G)
        S, Sa = c.scale * Q @ K.T, c.scale * abs(Q) @ abs(K).T
        if causal:
            S[np.arange(kT)[None, :] > np.arange(T)[:, None] + kT - T] = -np.inf
        some = np.isfinite(S).any(axis=1, keepdims=True)
        top = np.where(some, S.max(axis=1, keepdims=True), 0.0)
        P = np.exp(S - top)
        total = np.where(some, P.sum(axis=1, keepdims=True), 1.0)
        P = P / total
        lse = top + np.log(total)
        O = P @ V
        dP, dPa = W @ V.T, abs(W) @ abs(V).T
        d, da = (W * O).sum(1, keepdims=True), abs(W * O).sum(1, keepdims=True)
        dS = P * (dP - d)
        size = np.where(np.isfinite(S), abs(S), 0.0) + abs(lse) + abs(top) + 1
        eP = ((2 * (dh + 8) * Sa + kT + 64 + 8 * size) * u + 2.0 ** -20) * (P > 0)
        ed = (dh + 8) * u * da
        eS = abs(dS) * (1.1 * 2.0 ** -16 + eP) + P * ((dh + 8) * u * dPa + ed)
        eV = P * (1.1 * 2.0 ** -16 + eP)
        at, kv = slice(h * dh, (h + 1) * dh), slice(h // G * dh, (h // G + 1) * dh)
        out["O"][:, at] = O
        out["dq"][:, at] = c.scale * dS @ K
        err["dq"][:, at] = c.scale * (eS + 2 * kT * u * abs(dS)) @ abs(K)
        out["dk"][:, kv] += c.scale * dS.T @ Q
        err["dk"][:, kv] += c.scale * (eS + 2 * G * T * u * abs(dS)).T @ abs(Q)
        out["dv"][:, kv] += P.T @ W
        err["dv"][:, kv] += (eV + 2 * G * T * u * P).T @ abs(W)
    return out, err


def check(gpu, B, T, kT, G, Hk, dh, causal, names):
    torch, ql = gpu
    for seed in range(B):
        c = Case(torch, 1, T, Hk * G, Hk=Hk, kT=kT, dh=dh, causal=causal, seed=seed)
        out, err = exact(c, T, kT, G, Hk, dh, causal)
        _, lse = ql.attention_forward(c.q, c.k, c.v, *c.shape, **c.how)
        O = torch.from_numpy(out["O"].astype(np.float32)).cuda()
        g = ql.attention_backward(c.q, c.k, c.v, O, lse, c.dO, *c.shape, dtype=torch.float32,
                                  **c.how)
        for name, x in (("dq", g.q), ("dk", g.k), ("dv", g.v)):
            if name in names:
                off, bound = abs(host(x) - out[name]), err[name] + 1e-36
                assert (off <= bound).all(), (name, float((off / bound).max()))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T, kT, G, Hk", [(1, 479, 1, 4), (2, 557, 1, 4), (36, 560, 1, 1),
                                          (8, 245, 2, 2), (128, 129, 1, 2), (64, 300, 2, 1),
                                          (1, 3000, 8, 2), (31, 1500, 4, 3), (3, 193, 40, 2),
                                          (606, 606, 1, 1), (256, 140, 4, 2)])
def test_few_queries(gpu, T, kT, G, Hk, causal, dh):
    check(gpu, 2, T, kT, G, Hk, dh, causal, ("dq",))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T, kT, G, Hk", [(164, 15, 2, 1), (359, 5, 4, 2), (382, 29, 1, 1),
                                          (81, 81, 4, 1), (700, 128, 2, 2), (300, 1, 1, 2),
                                          (129, 127, 1, 3), (1500, 77, 1, 2),
                                          (606, 606, 1, 1), (140, 1024, 2, 2)])
def test_few_keys(gpu, T, kT, G, Hk, causal, dh):
    check(gpu, 2, T, kT, G, Hk, dh, causal, ("dk", "dv"))
