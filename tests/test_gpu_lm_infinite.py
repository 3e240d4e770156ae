"""Infinite weights, inputs and gradients in bf16: an infinite factor times a value that bf16 holds exactly, and times
one that it does not, is infinite with the product's sign; nothing but 0 times infinity, and infinities of
both signs, makes NaN.  The 64-bit form's pattern of infinities and NaN is exact; finite entries are not compared
beyond 2^-7 of their terms here (the operators' own tests do that)."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64
from tests.test_gpu_lora import adapters, order, rows
from tests.test_gpu_moe_few import params

pytestmark = pytest.mark.gpu
INF = float("inf")


def same_pattern(got, ref, what):
    got = np64(got)
    fin = np.isfinite(ref)
    odd = np.where(fin, ~np.isfinite(got), ~((got == ref) | (np.isnan(got) & np.isnan(ref))))
    assert not odd.any(), (what, odd.sum(), np.argwhere(odd)[:4], got[odd][:4], ref[odd][:4])
    assert (np.abs(got[fin] - ref[fin]) <= 2.0 ** -7 * (np.abs(ref[fin]).max() if fin.any() else 0)).all(), what


@pytest.mark.parametrize("n", [1, 5, 40])
def test_infinite_weights_of_an_expert(n):
    """h of small integers (one bf16 number) and of products (two); W2 with infinities in some columns of some rows."""
    K, d, h, o = 4, 264, 520, 264
    for exact in (True, False):
        p = params(K, d, h, o, "bf16", "relu", False, 3)
        g = torch.Generator().manual_seed(n)
        X = torch.randint(0, 2, (n, d), generator=g).bfloat16().cuda()
        if exact:
            p["W1"].copy_(torch.randint(-1, 2, p["W1"].shape, generator=g).bfloat16() * (torch.rand(p["W1"].shape, generator=g) < 0.1))
        p["W2"][:, 3, 5], p["W2"][:, 9, 7], p["W2"][:, 100, 11] = INF, -INF, INF
        p["W2"][:, 100, 13], p["W1"][1, 17] = -INF, INF
        f = hmoe.moe_few(p, X)
        e = f["expert"][:, 0].cpu().numpy()
        x, W1, W2 = np64(X), np64(p["W1"]), np64(p["W2"])
        with np.errstate(all="ignore"):
            hid = [W1[e[i]] @ x[i] for i in range(n)]
            hid = [np.where(v < 0, 0, v) for v in hid]
            ref = np.stack([W2[e[i]] @ hid[i] for i in range(n)])
        if n == 40:
            assert np.isposinf(ref).any() and np.isneginf(ref).any()
        same_pattern(f["Y"], ref, "Y")


@pytest.mark.parametrize("n,E,d,o,r", [(1, 3, 136, 72, 8), (40, 3, 136, 72, 24), (40, 3, 72, 16392, 40)])
@pytest.mark.parametrize("where", ["A", "B", "X"])
def test_infinite_adapters_of_few_rows(n, E, d, o, r, where):
    p, X, ids = integers(n, E, d, o, r, where)
    Y = hmoe.lora_few(p, X, torch.tensor(ids).cuda())
    same_pattern(Y, plain(p, X, ids, None)["Y"], "Y")


@pytest.mark.parametrize("n,E,d,o,r", [(40, 3, 136, 72, 24), (700, 3, 72, 136, 8), (16500, 3, 1032, 136, 24),
                                       (9000, 3, 264, 2312, 40)])
@pytest.mark.parametrize("where", ["A", "B", "X", "dY"])
def test_infinite_adapters_and_gradients_of_many_rows(n, E, d, o, r, where):
    p, X, ids = integers(n, E, d, o, r, where)
    dY = torch.randint(-1, 2, (n, o), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    if where == "dY":
        dY[2, 5] = INF
    off, perm = order(ids, E)
    Xs = X[perm.long()].contiguous()
    f = hmoe.lora_forward(p, Xs, off, perm)
    g = hmoe.lora_backward(p, Xs, off, dY, f["U"], perm)
    ref = plain(p, X, ids, dY)
    for k, v in {"Y": f["Y"], "dX": g["dX"], "dA": g["dA"], "dB": g["dB"]}.items():
        same_pattern(v, ref[k], k)


def integers(n, E, d, o, r, where):
    """Small integers, so that the narrow products are single bf16 numbers, with one infinity."""
    p = adapters(E, d, o, r, "bf16", True, 1, scale=False)
    g = torch.Generator().manual_seed(2)
    draw = lambda t: t.copy_(torch.randint(-1, 2, t.shape, generator=g).bfloat16() * (torch.rand(t.shape, generator=g) < 0.2))
    draw(p["A"]), draw(p["B"])
    X = rows(n, d, "bf16", 3)
    X.copy_(torch.randint(-1, 2, X.shape, generator=g).bfloat16())
    ids = (np.arange(n) % (E + 1) - 1).astype(np.int32)
    ids[0] = 1
    if where == "A":
        p["A"][1, 2, 3] = INF
    elif where == "B":
        p["B"][1, 7, :4] = INF
        p["B"][1, 9, 5] = -INF
    elif where == "X":
        X[0, 4] = -INF
    return p, X, ids


def plain(p, X, ids, dY):
    x, W, A, B, b = (np64(p[k]) if k != "X" else np64(X) for k in ("X", "W", "A", "B", "b"))
    with np.errstate(all="ignore"):
        out = {"Y": x @ W.T + b}
        if dY is not None:
            dy = np64(dY)
            out.update(dX=dy @ W, dA=np.zeros(A.shape), dB=np.zeros(B.shape))
        for e in range(A.shape[0]):
            i = np.nonzero(ids == e)[0]
            u = x[i] @ A[e].T
            out["Y"][i] += u @ B[e].T
            if dY is not None:
                v = dy[i] @ B[e]
                out["dX"][i] += v @ A[e]
                out["dA"][e], out["dB"][e] = v.T @ x[i], dy[i].T @ u
    return out


def test_sums_of_integers_are_exact():
    """Nothing of how a value is taken apart shows in a product: of integers Y is exact, zeros too."""
    K, d, h, o, n = 4, 264, 520, 264, 40
    g = torch.Generator().manual_seed(4)
    few = lambda *s: (torch.randint(-1, 2, s, generator=g) * (torch.rand(s, generator=g) < 0.1)).bfloat16().cuda()
    p = params(K, d, h, o, "bf16", "relu", False, 3)
    p["W1"].copy_(few(K, h, d)), p["W2"].copy_(few(K, o, h))
    X = torch.randint(-1, 2, (n, d), generator=g).bfloat16().cuda()
    f = hmoe.moe_few(p, X)
    e, x, W1, W2 = f["expert"][:, 0].cpu().numpy(), np64(X), np64(p["W1"]), np64(p["W2"])
    ref = np.stack([W2[e[i]] @ np.maximum(W1[e[i]] @ x[i], 0) for i in range(n)])
    assert (ref == 0).any() and np.array_equal(np64(f["Y"]), np64(torch.tensor(ref).bfloat16()))
    E, r = 3, 24
    for m in (1, n):
        q = {"W": few(o, d), "b": None, "A": few(E, r, d), "B": few(E, o, r), "scale": None}
        ids = np.arange(m).astype(np.int32) % E
        ref = plain(dict(q, b=torch.zeros(o)), X[:m], ids, None)["Y"]
        want = np64(torch.tensor(ref).bfloat16())
        assert (ref == 0).any() and np.array_equal(np64(hmoe.lora_few(q, X[:m], torch.tensor(ids).cuda())), want)
        off, perm = order(ids, E)
        assert np.array_equal(np64(hmoe.lora_forward(q, X[:m][perm.long()].contiguous(), off, perm)["Y"]), want)
