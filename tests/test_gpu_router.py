"""The learned router of a batch and its gradients against the formulas in 64 bits.

Bounds.  A score of d products is summed in fp32 with d / 4 additions one after the other at most: off by
(d / 4 + 8) 2^-24 sum |R| |x|.  Everything behind it is checked from the scores that the call returned, in 64 bits: choices
are equal; exp of a difference of scores of at most 64 is good to (64 + 4) 2^-24, and a probability, with its sum, to
160 2^-24.  The scores' gradient is off by 320 2^-24 of the magnitudes of its terms, and its products with R and X by
(K / 4 + 8) and (rows / 4 + 128) 2^-24 of theirs on top, dX of bf16 data by 2^-16 more and its rounding."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64, npi

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def make(n, K, d, dtype, seed=0, spread=2.0, off=()):
    g = torch.Generator(device="cuda").manual_seed(seed)
    R = (torch.randn(K, d, generator=g, device="cuda") * spread * d ** -0.5).to(DT[dtype])
    b = torch.randn(K, generator=g, device="cuda") * 0.3
    for e in off:
        b[e] = float("-inf")
    X = torch.randn(n, d, generator=g, device="cuda").to(DT[dtype])
    return {"R": R, "bias": b}, X, g


def soft(s):
    """Probabilities and ln sum exp; rows of -inf alone give zeros and 0."""
    mx = s.max(1, keepdims=True)
    none = np.isneginf(mx)
    e = np.where(none, 0.0, np.exp(s - np.where(none, 0.0, mx)))
    t = e.sum(1, keepdims=True)
    return e / np.where(none, 1.0, t), np.where(none, 0.0, mx + np.log(np.where(none, 1.0, t)))


def check_forward(f, X, p, top, renorm):
    n, K = f["scores"].shape
    R, b, x, s = np64(p["R"]), np64(p["bias"]) if p["bias"] is not None else np.zeros(K), np64(X), np64(f["scores"])
    ref = x @ R.T + b
    on = np.isfinite(b)
    assert np.isneginf(s[:, ~on]).all()
    mag = np.abs(x) @ np.abs(R[on]).T + np.abs(b[on])
    assert (np.abs(s[:, on] - ref[:, on]) <= (x.shape[1] / 4 + 8) * U * mag).all()
    idx = np.argsort(-s, axis=1, kind="stable")[:, :top]
    assert np.array_equal(npi(f["expert"]), idx)
    P, lse = soft(s)
    w = np.take_along_axis(P, idx, 1)
    if renorm:
        t = w.sum(1, keepdims=True)
        w = w / np.where(t == 0, 1.0, t)
    assert (np.abs(np64(f["weight"]) - w) <= 160 * U * w + 1e-37).all()
    real = np.isfinite(np.take_along_axis(s, idx, 1))
    counts = np.bincount(idx[real], minlength=K)
    assert np.array_equal(npi(f["counts"]), counts)
    share = P.mean(0)
    assert (np.abs(np64(f["share"]) - share) <= 256 * U * share + 1e-37).all()
    loss = np64(f["loss"])
    balance, z = K * (counts / (n * top) * share).sum(), (lse ** 2).mean()
    assert abs(loss[0] - balance) <= 300 * U * balance
    assert abs(loss[1] - z) <= 16 * U * (np.abs(lse) * (np.abs(lse) + np.abs(s[:, on]).max(initial=0.0))).mean() + 1e-12


def check_backward(g, f, X, p, top, renorm, gw, cb, cz, dtype):
    n, K = f["scores"].shape
    R, x, s, idx, counts = np64(p["R"]), np64(X), np64(f["scores"]), npi(f["expert"]), npi(f["counts"])
    P, lse = soft(s)
    rows = np.arange(n)[:, None]
    gw = np.zeros((n, top)) if gw is None else np64(gw)
    q = np.broadcast_to(cb * K * counts / (n * n * top), (n, K)).copy()
    mq = np.abs(q)
    if not renorm:
        np.add.at(q, (rows, idx), gw)
        np.add.at(mq, (rows, idx), np.abs(gw))
    zl = 2 * cz * lse / n
    ds = P * (q - (P * q).sum(1, keepdims=True) + zl)
    md = P * (mq + (P * mq).sum(1, keepdims=True) + np.abs(zl))
    if renorm:
        w = np.take_along_axis(P, idx, 1)
        t = w.sum(1, keepdims=True)
        w = w / np.where(t == 0, 1.0, t)
        np.add.at(ds, (rows, idx), w * (gw - (w * gw).sum(1, keepdims=True)))
        np.add.at(md, (rows, idx), w * (np.abs(gw) + (w * np.abs(gw)).sum(1, keepdims=True)))
    md = md * 320 * U + 1e-40
    dX, aR = ds @ R, np.abs(R)
    half = torch.finfo(DT[dtype]).eps / 2
    lim = half * np.abs(dX) + (1 + half) * (md @ aR + ((K / 4 + 8) * U + (2.0 ** -16 if dtype == "bf16" else 0)) * np.abs(ds) @ aR)
    assert (np.abs(np64(g["dX"]) - dX) <= lim + 1e-37).all()
    lim = md.T @ np.abs(x) + (n / 4 + 128) * U * np.abs(ds).T @ np.abs(x)
    assert (np.abs(np64(g["dR"]) - ds.T @ x) <= lim + 1e-37).all()
    lim = md.sum(0) + (n / 16 + 128) * U * np.abs(ds).sum(0)
    assert (np.abs(np64(g["dbias"]) - ds.sum(0)) <= lim + 1e-37).all()


CASES = [(1, 1, 8, 1), (5, 3, 24, 2), (64, 16, 64, 1), (777, 8, 64, 1), (130, 17, 72, 4), (300, 64, 200, 8), (257, 65, 136, 3),
         (500, 128, 264, 4), (129, 200, 1000, 2), (100, 256, 64, 8), (70, 300, 520, 2), (33, 1025, 64, 8), (17, 4096, 40, 5),
         (4000, 16, 1024, 2), (2000, 128, 520, 4),
         # scores and choices in one kernel; more tiles than workgroups
         (16500, 12, 40, 2), (17001, 30, 24, 8), (20000, 64, 72, 3), (18003, 100, 136, 4), (140001, 5, 8, 1), (70001, 70, 8, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("n,K,d,top", CASES)
def test_sizes(n, K, d, top, renorm, dtype):
    p, X, g = make(n, K, d, dtype, n + K)
    f = hmoe.router_forward(p, X, top_k=top, renorm=renorm)
    check_forward(f, X, p, top, renorm)
    gw = torch.randn(n, top, generator=g, device="cuda") / n
    b = hmoe.router_backward(p, X, f, gw, balance=0.3, z=0.2, renorm=renorm)
    check_backward(b, f, X, p, top, renorm, gw, 0.3, 0.2, dtype)


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("K,top", [(12, 3), (40, 4), (128, 8)])
def test_experts_that_are_off(K, top, renorm):
    off = [e for e in range(K) if e % 5 in (0, 3)]
    p, X, g = make(200, K, 64, "bf16", K, off=off)
    f = hmoe.router_forward(p, X, top_k=top, renorm=renorm)
    check_forward(f, X, p, top, renorm)
    gw = torch.randn(200, top, generator=g, device="cuda")
    b = hmoe.router_backward(p, X, f, gw, balance=1.0, z=0.5, renorm=renorm)
    check_backward(b, f, X, p, top, renorm, gw, 1.0, 0.5, "bf16")
    assert not b["dR"][off].any() and not b["dbias"][off].any()
    assert not f["counts"][off].any() and not f["share"][off].any()


def test_fewer_experts_than_choices_and_none():
    p, X, g = make(50, 10, 32, "f32", 3, off=[0, 1, 2, 3, 4, 5, 6, 8])
    f = hmoe.router_forward(p, X, top_k=4, renorm=True)  # two are on
    check_forward(f, X, p, 4, True)
    assert f["counts"].sum() == 100 and not f["weight"][:, 2:].any()
    gw = torch.randn(50, 4, generator=g, device="cuda")
    check_backward(hmoe.router_backward(p, X, f, gw, 1.0, 1.0, renorm=True), f, X, p, 4, True, gw, 1.0, 1.0, "f32")
    p["bias"].fill_(float("-inf"))
    f = hmoe.router_forward(p, X, top_k=4)
    check_forward(f, X, p, 4, False)
    for k in ("weight", "counts", "share", "loss"):
        assert not f[k].any(), k
    for renorm in (False, True):
        b = hmoe.router_backward(p, X, f, gw, 1.0, 1.0, renorm=renorm)
        for k in b:
            assert not b[k].any(), k


def test_equal_scores_go_to_the_lowest_experts():
    p, X, _ = make(64, 96, 64, "bf16")
    p["R"][:] = p["R"][:1]
    p["bias"] = None
    f = hmoe.router_forward(p, X, top_k=8)
    assert (f["expert"] == torch.arange(8, device="cuda")).all()
    check_forward(f, X, p, 8, False)


def test_not_numbers():
    p, X, _ = make(40, 20, 64, "bf16")
    clean = hmoe.router_forward(p, X, top_k=3)
    X[7, 3] = float("nan")
    f = hmoe.router_forward(p, X, top_k=3)
    keep = [i for i in range(40) if i != 7]
    for k in ("expert", "weight", "scores"):
        assert torch.equal(f[k][keep], clean[k][keep])
    assert torch.isnan(f["weight"][7]).all() and (f["expert"][7] == torch.arange(3, device="cuda")).all()
    assert torch.isnan(f["loss"]).all() and torch.isnan(f["share"]).all()
    assert f["counts"].sum() == 39 * 3
    for renorm in (False, True):
        b = hmoe.router_backward(p, X, f, torch.ones(40, 3, device="cuda"), 1.0, 1.0, renorm=renorm)
        assert not torch.isnan(b["dX"][7].float()).logical_not().any()
    # experts that are off rank above one of NaN, and the rows have NaN for weights all the same
    p["bias"][1:] = float("-inf")
    p["R"][0] = float("nan")
    X[7] = 0
    f = hmoe.router_forward(p, X, top_k=3, renorm=True)
    assert (f["expert"] == torch.tensor([1, 2, 3], device="cuda")).all() and torch.isnan(f["weight"]).all()
    assert not f["counts"].any() and torch.isnan(f["loss"]).all()
    b = hmoe.router_backward(p, X, f, torch.ones(40, 3, device="cuda"), 1.0, 1.0, renorm=True)
    assert torch.isnan(b["dX"].float()).all()


def test_no_rows_and_what_is_not_wanted():
    p, X, _ = make(0, 12, 64, "f32")
    f = hmoe.router_forward(p, X, top_k=2)
    for k in ("counts", "share", "loss"):
        assert not f[k].any()
    b = hmoe.router_backward(p, X, f, balance=1.0)
    assert b["dX"].shape == (0, 64) and not b["dR"].any() and not b["dbias"].any()
    p, X, g = make(90, 12, 64, "f32")
    f = hmoe.router_forward(p, X, top_k=2)
    gw = torch.randn(90, 2, generator=g, device="cuda")
    whole = hmoe.router_backward(p, X, f, gw, 0.1, 0.1)
    one = hmoe.router_backward(p, X, f, gw, 0.1, 0.1, want_dX=False)
    two = hmoe.router_backward(p, X, f, gw, 0.1, 0.1, want_router=False)
    assert one["dX"] is None and two["dR"] is None
    assert torch.equal(one["dR"], whole["dR"]) and torch.equal(one["dbias"], whole["dbias"]) and torch.equal(two["dX"], whole["dX"])
    none = hmoe.router_backward(p, X, f)
    assert not none["dX"].any() and not none["dR"].any()


def test_the_same_choices_as_the_layer_of_a_few_samples():
    g = torch.Generator(device="cuda").manual_seed(2)
    p, X, _ = make(60, 24, 64, "f32", 9)
    w = lambda *s: torch.randn(*s, generator=g, device="cuda") * 0.1
    few = hmoe.moe_few({"R": p["R"], "r_bias": p["bias"], "W1": w(24, 32, 64), "b1": None, "W2": w(24, 16, 32), "b2": None},
                       X, top_k=3)
    f = hmoe.router_forward(p, X, top_k=3, renorm=True)
    s = np.sort(np64(f["scores"]), 1)[:, ::-1]
    clear = torch.tensor((s[:, :3] - s[:, 1:4] > 1e-4).all(1), device="cuda")
    assert clear.sum() > 40
    assert torch.equal(f["expert"][clear], few["expert"][clear])
    assert (f["weight"] - few["weight"])[clear].abs().max() <= 1e-5


def test_against_differences():
    """The gradient along random directions from differences in 64 bits of the formulas, counts fixed."""
    n, K, d, top = 30, 9, 16, 2
    p, X, g = make(n, K, d, "f32", 4)
    gw = torch.randn(n, top, generator=g, device="cuda")
    for renorm in (False, True):
        f = hmoe.router_forward(p, X, top_k=top, renorm=renorm)
        b = hmoe.router_backward(p, X, f, gw, 2.0, 0.7, renorm=renorm)
        idx, counts = npi(f["expert"]), npi(f["counts"])

        def value(x, R, bias):
            P, lse = soft(x @ R.T + bias)
            w = np.take_along_axis(P, idx, 1)
            if renorm:
                w = w / w.sum(1, keepdims=True)
            return (w * np64(gw)).sum() + 2.0 * K * (counts / (n * top) * P.mean(0)).sum() + 0.7 * (lse ** 2).mean()

        at = [np64(X), np64(p["R"]), np64(p["bias"])]
        rs = np.random.default_rng(1)
        for i, key in enumerate(("dX", "dR", "dbias")):
            v = rs.standard_normal(at[i].shape)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
            want, got = (value(*up) - value(*down)) / 2e-5, (np64(b[key]) * v).sum()
            assert abs(got - want) <= 1e-4 * np.abs(np64(b[key]) * v).sum(), (renorm, key, got, want)


def test_captured_and_replayed():
    n, K, d, top = 300, 20, 128, 2
    p, X, g = make(n, K, d, "bf16")
    gw = torch.randn(n, top, generator=g, device="cuda")
    want_f = hmoe.router_forward(p, X, top_k=top)
    want_b = hmoe.router_backward(p, X, want_f, gw, 0.1, 0.1)
    of, ob = {k: torch.empty_like(v) for k, v in want_f.items()}, {k: torch.empty_like(v) for k, v in want_b.items()}
    ws = torch.empty(hmoe.router_workspace(p, n, top), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hmoe.router_forward(p, X, top_k=top, out=of, ws=ws)
        hmoe.router_backward(p, X, of, gw, 0.1, 0.1, out=ob, ws=ws)
    for _ in range(3):
        for t in (*of.values(), *ob.values()):
            t.fill_(3)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in ((of, want_f), (ob, want_b)):
            for k in want:
                assert torch.equal(got[k], want[k]), k
