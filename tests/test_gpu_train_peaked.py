"""The masked attention where a row's probability is that of a few keys (scores of a large
spread): errors of whole tensors, where the bounds element by element leave room for
roundings that all agree.

A rounding to bf16 is off by 2^-8 / sqrt(3) = U of its value in the root of the mean square
at most (evenly spread over up to half a step, at the worst place between two powers of two),
and roundings are independent of each other.
  O = sum p_j V_j / sum p_j over rounded p_j is a mean with weights that are off by e_j P_j:
      it is off by sum e_j P_j (V_j - O), U of its norm or less; its own rounding is another U.
  dS rounded, and d = <dO, O> off by sum e_j P_j (dP_j - d) = sum e_j dS_j: the first is
      off by sum e'_j dS_j K_j in dq, the second by (sum e_j dS_j) (sum P_j K_j), no more where
      the K_j are of one size: U each; the output's own rounding is a third.  (In dk the same
      with Q.)  dv: P rounded, and the output.
  An O that is kept in bf16: d off by sum over channels of e_c dO_c O_c besides, which no
      smallness of dS lessens."""
import numpy as np
import pytest

from test_gpu_train_attention import host

pytestmark = pytest.mark.gpu

U = 2.0 ** -8 / 3 ** 0.5


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def exact(q, k, v, dO, H, Hk, dh, causal):
    """O, dq, dk, dv in 64 bits, and what a bf16 O costs dq and dk (root of the sum of
    squares)."""
    T, kT, G, scale = q.shape[0], k.shape[0], H // Hk, dh ** -0.5
    out = [np.zeros_like(x) for x in (q, q, k, v)]
    cost = [0.0, 0.0]
    see = np.ones((T, kT), bool)
    if causal:
        see = np.arange(kT)[None, :] <= np.arange(T)[:, None] + kT - T
    for h in range(H):
        a, b = slice(h * dh, (h + 1) * dh), slice(h // G * dh, (h // G + 1) * dh)
        Q, K, V, D = q[:, a], k[:, b], v[:, b], dO[:, a]
        S = np.where(see, Q @ K.T * scale, -np.inf)
        P = np.exp(S - S.max(axis=1, keepdims=True))
        P /= P.sum(axis=1, keepdims=True)
        O = P @ V
        dS = P * (D @ V.T - (D * O).sum(axis=1, keepdims=True)) * scale
        out[0][:, a], out[1][:, a] = O, dS @ K
        out[2][:, b] += dS.T @ Q
        out[3][:, b] += P.T @ D
        d2 = (U * scale) ** 2 * ((D * O) ** 2).sum(axis=1)
        cost[0] += (d2 * ((P @ K) ** 2).sum(axis=1)).sum()
        cost[1] += ((P ** 2).T @ (d2 * (Q ** 2).sum(axis=1))).sum()
    return out, [0.0, *np.sqrt(cost), 0.0]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("std", [1, 4, 10, 30])
@pytest.mark.parametrize("T, kT, H, Hk", [(129, 129, 6, 6), (200, 600, 8, 2), (600, 600, 4, 4),
                                          (5, 2000, 16, 2)])
def test_errors_of_the_whole(gpu, T, kT, H, Hk, std, causal, dh):
    torch, ql = gpu
    rng = np.random.default_rng(T + kT + std)
    new = lambda n, heads, s: torch.from_numpy((rng.standard_normal((n, heads * dh)) * s).astype(
        np.float32)).to(torch.bfloat16).cuda()
    q, k, v, dO = new(T, H, std), new(kT, Hk, 1.0), new(kT, Hk, 1.0), new(T, H, 0.1)
    want, cost = exact(*(host(t) for t in (q, k, v, dO)), H, Hk, dh, causal)
    how = dict(kv_heads=Hk, dh=dh, kT=kT, causal=causal)
    for odtype in (torch.float32, torch.bfloat16):
        O, lse = ql.attention_forward(q, k, v, 1, T, H, odtype=odtype, **how)
        g = ql.attention_backward(q, k, v, O, lse, dO, 1, T, H, **how)
        kept = odtype == torch.bfloat16
        for name, got, x, n, more in zip(("O", "dq", "dk", "dv"), (O, *g), want,
                                         (1 + kept, 3, 3, 2), cost):
            size, off = np.linalg.norm(x), np.linalg.norm(host(got) - x)
            bound = (n * U ** 2 + (more / size) ** 2 * kept) ** 0.5
            print(name, str(odtype)[6:], "off by %.5f, bound %.5f" % (off / size, bound))
            assert off <= bound * size, (name, odtype, off / size, bound)
