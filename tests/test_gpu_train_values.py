"""The masked attention and what rows hold or where they lie: values that are not finite,
sequences on their own, offsets and lengths that leave the tensors."""
import numpy as np
import pytest

from test_gpu_train_attention import Case, compare, i64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (run with -m 'not gpu' on a CPU host)")
    from paper_2607_08526_amd import qlinear as ql
    ql.load()
    return torch, ql


def both(ql, c, **inputs):
    """O, lse, dq, dk, dv with some of q, k, v, dO in other tensors; O and lse of the
    case's own inputs enter the backward pass where only dO is another."""
    x = {n: inputs.get(n, getattr(c, n)) for n in ("q", "k", "v", "dO")}
    O, lse = ql.attention_forward(x["q"], x["k"], x["v"], *c.shape, **c.how)
    g = ql.attention_backward(x["q"], x["k"], x["v"], O, lse, x["dO"], *c.shape, **c.how)
    return dict(O=O, lse=lse.t(), dq=g.q, dk=g.k, dv=g.v)


def same(torch, a, b, rows, cols):
    return torch.equal(a[rows][:, cols], b[rows][:, cols])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lens, klens", [([70, 33, 5], [300, 64, 1]), ([260, 100, 300], None)],
                         ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_keep_to_their_rows(gpu, lens, klens, bad, dh):
    """A value that is not finite in a query, key, value or output gradient of one head of a
    sequence: the other sequences' and heads' results, and for a query the other queries',
    are the same to the bit; those that have to do with a NaN are NaN."""
    torch, ql = gpu
    H, Hk, G = 4, 2, 2
    c = Case(torch, 3, max(lens), H, Hk=Hk, dh=dh, kT=max(klens or lens), rows="packed", lens=lens,
             klens=klens)
    s, at = c.seqs[1], 7
    want = both(ql, c)
    for n in ("q", "dO", "k", "v"):
        query = n in ("q", "dO")
        t = getattr(c, n).clone()
        head = 2 if query else 1          # key head 1, query heads 2 and 3
        row = (s.q if query else s.k) + at
        t[row, head * dh + 3] = bad
        got = both(ql, c, **{n: t})
        for name, x in got.items():
            width = 1 if name == "lse" else dh
            keys = name in ("dk", "dv")
            first, n_rows = (s.k, s.m) if keys else (s.q, s.n)
            rows = torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
            rows[first: first + n_rows] = False
            assert same(torch, x, want[name], rows, slice(None)), (n, name)  # other sequences
            here = slice(first, first + n_rows)
            hit = [1] if keys else [2, 3]
            clean = [h for h in range(Hk if keys else H) if h not in hit]
            for h in clean:
                cols = slice(h * width, (h + 1) * width)
                assert same(torch, x, want[name], here, cols), (n, name)
            for h in hit:
                cols = slice(h * width, (h + 1) * width)
                if query and not keys:  # the query's own row alone, of its own head
                    for r in [i for i in range(first, first + n_rows) if i != row or h != head]:
                        assert same(torch, x, want[name], slice(r, r + 1), cols), (n, name, r)
                    touched = x[row: row + 1, cols] if h == head else None
                    if n == "dO" and name in ("O", "lse"):
                        touched = None
                else:
                    touched = x[here, cols]
                    if (n, name) in (("v", "lse"), ("v", "dv"), ("dO", "O"), ("dO", "lse")):
                        assert torch.equal(touched, want[name][here, cols])
                        touched = None
                    if (n, name) in (("dO", "dv"), ("v", "O")):  # that channel alone
                        rest = [i for i in range(dh) if i != 3]
                        assert torch.equal(touched[:, rest], want[name][here, cols][:, rest])
                        touched = touched[:, 3]
                if touched is not None and bad != bad:
                    assert torch.isnan(touched).all(), (n, name)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("shift", [0, -90, 57])
def test_reach_of_what_the_causal_mask_hides(gpu, shift, bad, dh):
    """Under a causal mask a value that is not finite may reach rows beside those that see
    it, but not 256 away: the queries before, and in the gradients of k and v the keys
    behind."""
    torch, ql = gpu
    T = 900
    c = Case(torch, 2, T, 2, Hk=1, dh=dh, kT=T + shift, causal=True)
    want = both(ql, c)
    for at in (517, 640, 701):
        for n in ("k", "v"):
            t = getattr(c, n).clone()
            t[at] = bad
            got = both(ql, c, **{n: t})
            for name in ("O", "lse", "dq"):
                rows = torch.arange(got[name].shape[0], device="cuda")
                clean = (rows >= T) | (rows + shift <= at - 256)
                assert same(torch, got[name], want[name], clean, slice(None)), (n, name)
        for n in ("q", "dO"):
            t = getattr(c, n).clone()
            t[at] = bad
            got = both(ql, c, **{n: t})
            for name in ("dk", "dv"):
                rows = torch.arange(got[name].shape[0], device="cuda")
                clean = (rows >= T + shift) | (rows >= at + shift + 256)
                assert same(torch, got[name], want[name], clean, slice(None)), (n, name)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("how", [dict(lens=[200, 50, 131]),
                                 dict(lens=[130, 1, 64], klens=[9, 700, 64])], ids=str)
def test_sequences_alone(gpu, how, causal, dh):
    """Each sequence of a packed batch as it is on its own (its parts of the keys may be
    others: each is off by its bound)."""
    torch, ql = gpu
    lens, klens = how["lens"], how.get("klens", how["lens"])
    c = Case(torch, 3, max(lens), 4, Hk=2, dh=dh, kT=max(klens), rows="packed", causal=causal,
             **how)
    got, bounds = both(ql, c), c.want(grads=True)
    for s in c.seqs:
        q, k = slice(s.q, s.q + s.n), slice(s.k, s.k + s.m)
        args = (c.q[q], c.k[k], c.v[k])
        alone = dict(kv_heads=2, dh=dh, kT=s.m, causal=causal)
        O, lse = ql.attention_forward(*args, 1, s.n, 4, **alone)
        g = ql.attention_backward(*args, O, lse, c.dO[q], 1, s.n, 4, **alone)
        for name, x, rows in (("O", O, q), ("lse", lse.t(), q), ("dq", g.q, q), ("dk", g.k, k),
                              ("dv", g.v, k)):
            bound = bounds[name][1].T if name == "lse" else bounds[name][1]
            a, b = (t.double().cpu().numpy() for t in (x, got[name][rows]))
            with np.errstate(invalid="ignore"):
                assert ((np.abs(a - b) <= 2 * bound[rows]) | (a == b)).all(), name


def clamped(offsets, lens, rows, T):
    """The rows that each sequence's place has, by the rule that the header states."""
    for b in range(len(offsets) - 1):
        lo = min(max(offsets[b], 0), rows)
        hi = min(max(offsets[b + 1], lo), rows)
        cap = min(hi - lo, T)
        yield lo, cap, cap if lens is None else min(max(lens[b], 0), cap)


BAD = [([0, 10 ** 12, -5, 2], None), ([150, 0, 150, 150], None), ([-7, -3, -1, -1], None),
       ([40, 90, 60, 100], [10 ** 15, -1, 7]),
       ([0, 30, 30, 5 * 10 ** 18], [-(10 ** 18), 3, 10 ** 9])]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("offsets, lens", BAD, ids=str)
def test_offsets_out_of_place(gpu, offsets, lens, causal, dh):
    """Offsets that fall or leave the tensor, lengths below zero and past their place: nothing
    is written but the rows that the header's rule leaves, in outputs that lie between
    others' rows and columns."""
    torch, ql = gpu
    rows, T, H, Hk, guard = 150, 90, 2, 1, 200
    c = Case(torch, 3, T, H, Hk=Hk, dh=dh, causal=causal, rows="packed", lens=[rows // 3] * 3)
    q, k, v, dO = (torch.randn((rows, n * dh), device="cuda").to(torch.bfloat16)
                   for n in (H, Hk, Hk, H))
    how = c.how | dict(q_offsets=i64(torch, offsets), k_offsets=i64(torch, offsets))
    if lens is not None:
        how |= dict(q_lens=i64(torch, lens), k_lens=i64(torch, lens))
    place = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for lo, cap, _ in clamped(offsets, lens, rows, T):
        place[lo: lo + cap] = True
    whole, views = [], []
    for n in (H, H, Hk, Hk):
        whole.append(torch.full((rows + 2 * guard, n * dh + 16), 7.0, dtype=torch.bfloat16,
                                device="cuda"))
        views.append(whole[-1][guard: guard + rows, 8: 8 + n * dh])
    sums = torch.full((H * rows + 2 * guard,), 7.0, device="cuda")
    lse = sums[guard: guard + H * rows].view(H, rows)
    O, dq, dk, dv = views
    ql.attention_forward(q, k, v, 3, T, H, O=O, lse=lse, **how)
    ql.attention_backward(q, k, v, O, lse, dO, 3, T, H, dq=dq, dk=dk, dv=dv, **how)
    torch.cuda.synchronize()
    for w, x in zip(whole, views):
        assert (w[:guard] == 7).all() and (w[guard + rows:] == 7).all()
        assert (w[:, :8] == 7).all() and (w[:, -8:] == 7).all()
        assert (x[~place] == 7).all() and not (x[place] == 7).all(dim=1).any()
    assert (sums[:guard] == 7).all() and (sums[guard + H * rows:] == 7).all()
    assert (lse[:, ~place] == 7).all()
