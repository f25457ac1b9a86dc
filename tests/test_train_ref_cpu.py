"""The 64-bit references of the training operators (train_ref.py) on the CPU: their
gradients, which the GPU tests compare the kernels with element by element, against
differences of their own forward formulas and against torch's differentiation.

Differences: (f(x + t d) - f(x - t d)) / 2 t along unit directions d of all of a tensor, t =
1e-4.  Off by t^2 / 6 = 1.7e-9 of a third derivative (of the order of the first, as scores
and normalised values move by at most a few t) and by 2^-53 |f| / t, 1e-12 |f|.  Held to 1e-6
of the gradient's norm: along the gradient itself the derivative is that norm, so a zero, a
sign or a factor that is wrong fails by far more, and along random directions, which have
about n^-1/2 of their length in each of n elements, so does a single element of average size
that is wrong by a hundredth (n up to 6000: 0.01 / n of the norm)."""
import numpy as np
import pytest
import torch

import train_ref as R

T_STEP = 1e-4


def agree(f, x, g, rng, directions=6):
    """f: the scalar of x; g: its gradient."""
    size = np.linalg.norm(g)
    assert size > 0
    for k in range(directions):
        d = g if k == 0 else rng.standard_normal(x.shape)
        d = d / np.linalg.norm(d)
        diff = (f(x + T_STEP * d) - f(x - T_STEP * d)) / (2 * T_STEP)
        if not abs((g * d).sum() - diff) <= 1e-6 * size:
            return False
    return True


CASES = [
    # sequences of (first, live, place) on both sides, H, Hk, dh, causal
    ([((0, 48, 48), (0, 60, 60))], 2, 1, 64, True),
    ([((0, 30, 30), (0, 30, 30))], 2, 2, 128, False),
    ([((2, 9, 11), (0, 20, 20)), ((13, 7, 7), (20, 3, 8))], 4, 2, 64, True),  # some see no key
    ([((0, 5, 5), (3, 1, 1)), ((5, 6, 9), (4, 33, 40))], 6, 2, 64, False),    # one key
]


def rows(case, rng):
    seqs, H, Hk, dh, causal = case
    qrows = max(q[0] + q[2] for q, _ in seqs) + 2
    krows = max(k[0] + k[2] for _, k in seqs) + 1
    new = lambda n, h: rng.standard_normal((n, h * dh))
    return [new(qrows, H), new(krows, Hk), new(krows, Hk)], new(qrows, H) * 0.3


def by_hand(case, x, dO):
    seqs, H, Hk, dh, causal = case
    out = R.attention(*x, [R.Seq(q, k) for q, k in seqs], H, Hk, dh, dh ** -0.5, causal, False, dO,
                      False)
    return {n: np.nan_to_num(v, nan=0.0) for n, (v, _) in out.items()}


@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_attention_gradients(case):
    rng = np.random.default_rng(3)
    x, dO = rows(case, rng)
    want = by_hand(case, x, dO)
    for i, name in enumerate(("dq", "dk", "dv")):
        def f(y):
            z = list(x)
            z[i] = y
            return (by_hand(case, z, dO)["O"] * dO).sum()
        g = want[name]
        assert agree(f, x[i], g, rng), name
        # what the check is for: each of these fails it
        one = g.copy()
        one[tuple(np.argwhere(np.abs(g) > np.abs(g).mean())[0])] *= 1.5
        for wrong in (-g, 0.999 * g, np.roll(g, 1, axis=1), np.roll(g, 1, axis=0)):
            assert not agree(f, x[i], wrong, rng), name
        assert not agree(f, x[i], one, rng, 12), name


@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_attention_by_torch(case):
    """Output, row sums and gradients by torch's softmax and differentiation in 64 bits."""
    seqs, H, Hk, dh, causal = case
    rng = np.random.default_rng(4)
    x, dO = rows(case, rng)
    want = by_hand(case, x, dO)
    leaves = [torch.from_numpy(t).requires_grad_() for t in x]
    total = 0.0
    for (q0, n, _), (k0, m, _) in seqs:
        for h in range(H):
            a, b = slice(h * dh, (h + 1) * dh), slice(h * Hk // H * dh, (h * Hk // H + 1) * dh)
            for i in range(n):
                keys = min(m, i + m - n + 1) if causal else m
                if keys <= 0:
                    assert (want["O"][q0 + i, a] == 0).all()
                    assert want["lse"][h, q0 + i] < -1e300  # (-infinity)
                    continue
                K, V = (t[k0: k0 + keys, b] for t in leaves[1:])
                s = K @ leaves[0][q0 + i, a] / dh ** 0.5
                o = torch.softmax(s, 0) @ V
                assert np.abs(o.detach().numpy() - want["O"][q0 + i, a]).max() <= 1e-13
                assert abs(torch.logsumexp(s, 0).item() - want["lse"][h, q0 + i]) <= 1e-13
                total = total + (o * torch.from_numpy(dO[q0 + i, a])).sum()
    for name, g in zip(("dq", "dk", "dv"), torch.autograd.grad(total, leaves)):
        assert np.abs(g.numpy() - want[name]).max() <= 1e-13 * max(1.0, np.abs(want[name]).max())


@pytest.mark.parametrize("eps", [0.0, 1e-6, 0.5])
def test_norm_gradients(eps):
    rng = np.random.default_rng(5)
    h, dy, dres = (rng.standard_normal((7, 50)) for _ in range(3))
    w = 1 + 0.3 * rng.standard_normal(50)
    dx, dw, _, _ = R.norm_grads(dy, h, w, eps, dres)
    f = lambda y: (R.norm(y, w, eps) * dy).sum() + (y * dres).sum()
    assert agree(f, h, dx, rng)
    assert not agree(f, h, dx - dres, rng) and not agree(f, h, np.roll(dx, 1, axis=1), rng)
    f = lambda y: (R.norm(h, y, eps) * dy).sum()
    assert agree(f, w, dw, rng)
    assert not agree(f, w, -dw, rng)
