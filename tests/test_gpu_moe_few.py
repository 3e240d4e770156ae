"""The whole mixture layer for a few samples against a plain evaluation in 64 bits.

Tolerances (u = 2^-24).  A sum of N fp32 products, in chains of at most N / 16 + 16 additions (a lane's or an
MFMA's share, then the joins), is off by at most c(N) = (N / 16 + 16) u times the sum of the terms' absolute
values.  Scores: c(d); a softmax weight follows with twice the largest score error, relative, and 1e-6 for its
exponentials.  h: c(d) of its own terms through an activation of slope <= 1.1, 1e-6 relative for its
exponential, 2^-16 relative for the two bf16 numbers it is split into; the second layer passes those on
through |W2| and adds c(h).  bf16 outputs are rounded once: 2^-8 relative covers half an ulp.  Experts are
exact: samples whose deciding scores lie within the error are not drawn."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from paper_1704_06363_amd import workloads as W
from tests.parity import np64, npi

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24


def c(N):
    return (N / 16 + 16) * U


def params(K, d, h, o, dtype, act, bias, seed):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    rows = 2 * h if act == "silu" else h
    r = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dt).cuda()
    return {"R": r(K, d, std=d ** -0.5), "r_bias": (torch.randn(K, generator=g) * 0.1).cuda(),
            "W1": r(K, rows, d, std=d ** -0.5), "W2": r(K, o, h, std=h ** -0.5),
            "b1": r(K, rows, std=0.2) if bias else None, "b2": r(K, o, std=0.2) if bias else None}


def draw(p, n, k, dtype, seed, std=1.0):
    """n samples whose first k + 1 scores are apart."""
    d = p["R"].shape[1]
    g = torch.Generator().manual_seed(seed)
    X = (torch.randn(4 * n + 8, d, generator=g) * std).to(DT[dtype])
    s = np64(X) @ np64(p["R"]).T + np64(p["r_bias"])
    top = -np.sort(-s, axis=1)[:, :k + 1]
    with np.errstate(invalid="ignore"):
        ok = ~(np.diff(-top, axis=1) < 1e-3).any(1)
    return X[np.nonzero(ok)[0][:n]].cuda()


def plain(p, X, k, act):
    x, R, W1, W2 = (np64(t) for t in (X, p["R"], p["W1"], p["W2"]))
    K, o, h = W2.shape
    b1 = np64(p["b1"]) if p["b1"] is not None else np.zeros(W1.shape[:2])
    b2 = np64(p["b2"]) if p["b2"] is not None else np.zeros((K, o))
    rb = np64(p["r_bias"]) if p["r_bias"] is not None else np.zeros(K)
    s = x @ R.T + rb
    es = c(R.shape[1]) * (np.abs(x) @ np.abs(R).T)
    e = np.argsort(-s, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(s, e, 1)
    with np.errstate(all="ignore"):
        w = np.where(top == -np.inf, 0.0, np.exp(top - top[:, :1]))
    sw = w.sum(1, keepdims=True)
    w = np.where(sw > 0, w / np.where(sw > 0, sw, 1), 0.0)
    w = np.where(w < 2.0 ** -126, 0.0, w)  # by definition
    wt = w * (2 * np.take_along_axis(es, e, 1).max(1, keepdims=True) + 1e-6)
    n = len(x)
    Y, tol = np.zeros((n, o)), np.zeros((n, o))
    for i in range(n):
        for j in range(k):
            if w[i, j] == 0:
                continue
            q = e[i, j]
            z = W1[q] @ x[i] + b1[q]
            ez = c(x.shape[1]) * (np.abs(W1[q]) @ np.abs(x[i]) + np.abs(b1[q]))
            if act == "silu":
                g, up = z[:h], z[h:]
                with np.errstate(over="ignore"):
                    a = g / (1 + np.exp(-g))
                hid = a * up
                eh = (1.1 * ez[:h] + 1e-6 * np.abs(a)) * (np.abs(up) + ez[h:]) + np.abs(a) * ez[h:]
            else:
                hid, eh = np.maximum(z, 0), ez
            eh = eh + 2.0 ** -16 * np.abs(hid)
            y = W2[q] @ hid + b2[q]
            ey = np.abs(W2[q]) @ (eh + c(h) * np.abs(hid)) + c(h) * np.abs(b2[q])
            Y[i] += w[i, j] * y
            tol[i] += w[i, j] * (ey + 4 * U * np.abs(y)) + wt[i, j] * np.abs(y)
    return e, w, wt, Y, tol


def check(p, X, k, act, rows=slice(None)):
    f = hmoe.moe_few(p, X, top_k=k, act=act)
    torch.cuda.synchronize()
    e, w, wt, Y, tol = plain(p, X[rows], k, act)
    assert np.array_equal(npi(f["expert"])[rows], e)
    assert (np.abs(np64(f["weight"])[rows] - w) <= wt).all()
    if X.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(Y)
    off = ~(np.abs(np64(f["Y"])[rows] - Y) <= tol)
    assert not off.any(), (np.argwhere(off)[:4], np64(f["Y"])[rows][off][:4], Y[off][:4], tol[off][:4])
    return f


@pytest.mark.parametrize("dtype,n,K,d,h,o,k,act,bias", [
    ("f32", 1, 1, 8, 8, 8, 1, "relu", False), ("bf16", 1, 2, 8, 8, 8, 2, "silu", True),
    ("f32", 5, 8, 64, 128, 64, 1, "relu", True), ("bf16", 3, 16, 1000, 520, 136, 1, "relu", False),
    ("bf16", 16, 4, 136, 72, 200, 3, "silu", True), ("f32", 17, 5, 72, 40, 24, 5, "silu", False),
    ("bf16", 33, 3, 256, 264, 512, 1, "silu", False), ("bf16", 64, 128, 512, 256, 128, 4, "silu", True),
    ("f32", 64, 2, 96, 88, 104, 1, "relu", True), ("bf16", 64, 64, 64, 48, 40, 8, "relu", False),
    ("bf16", 2, 4096, 16, 8, 16, 8, "relu", True), ("f32", 64, 4096, 8, 16, 8, 2, "silu", False),
    ("bf16", 1, 16, 2048, 4096, 1024, 1, "relu", False), ("bf16", 8, 32, 2048, 1024, 1024, 2, "silu", True),
    ("f32", 9, 16, 1032, 1048, 520, 2, "silu", True)])
def test_sizes_types_and_choices(dtype, n, K, d, h, o, k, act, bias):
    p = params(K, d, h, o, dtype, act, bias, K + d)
    check(p, draw(p, n, k, dtype, n + h), k, act)


@pytest.mark.parametrize("dtype,K,d,h,o,k,act", [
    ("bf16", 64, 1032, 2056, 520, 4, "silu"), ("f32", 9, 520, 1032, 72, 8, "relu"), ("bf16", 700, 264, 520, 24, 1, "relu")])
def test_one_sample(dtype, K, d, h, o, k, act):
    """Its choices are groups of their own, their reductions split and joined."""
    p = params(K, d, h, o, dtype, act, True, K)
    check(p, draw(p, 1, k, dtype, 3), k, act)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_sample_with_one_expert(dtype):
    p = params(9, 200, 136, 72, dtype, "relu", True, 3)
    p["r_bias"][:] = 0
    p["r_bias"][6] = 100.0
    f = check(p, draw(p, 64, 1, dtype, 2), 1, "relu")
    assert (npi(f["expert"]) == 6).all()
    X = draw(p, 41, 2, dtype, 5)
    check(p, X, 2, "relu")


def test_equal_scores_go_to_the_lowest_expert():
    p = params(12, 64, 32, 40, "bf16", "relu", False, 4)
    p["R"][:] = p["R"][3].clone()
    p["r_bias"][:] = 0.5
    f = check(p, torch.randn(10, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda(), 4, "relu")
    assert (npi(f["expert"]) == np.arange(4)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_experts_that_are_off(dtype):
    p = params(10, 72, 48, 56, dtype, "silu", True, 5)
    p["r_bias"][3:] = float("-inf")
    p["W1"][3:] = float("nan")  # not evaluated: nothing of them may arrive
    p["W2"][3:] = float("inf")
    X = draw(p, 20, 3, dtype, 6)
    f = check(p, X, 5, "silu")  # two choices of weight 0
    assert (np64(f["weight"])[:, 3:] == 0).all()
    p["r_bias"][:] = float("-inf")
    f = hmoe.moe_few(p, X, top_k=3, act="silu")
    assert (np64(f["Y"]) == 0).all() and (np64(f["weight"]) == 0).all()
    assert (npi(f["expert"]) == np.arange(3)).all()


def test_lowest_value_as_a_mask():
    p = params(10, 72, 48, 56, "bf16", "relu", True, 7)
    p["r_bias"][4:] = torch.finfo(torch.float32).min / 2
    f = check(p, draw(p, 9, 2, "bf16", 8), 2, "relu")
    assert (npi(f["expert"]) < 4).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_bad_sample_stays_alone(value):
    p = params(6, 64, 48, 40, "bf16", "relu", True, 9)
    X = draw(p, 19, 2, "bf16", 10)
    X[7, 5] = value
    keep = np.arange(19) != 7
    f = check(p, X, 2, "relu", rows=torch.tensor(keep))
    e = npi(f["expert"])[7]
    assert (e >= 0).all() and (e < 6).all() and e[0] != e[1]
    assert np.isnan(np64(f["Y"])[7]).all()


def test_large_hidden_values_stay_finite():
    p = params(2, 8, 8, 8, "bf16", "relu", False, 2)
    p["W1"][:] = 1.0
    p["W2"][:] = 1.0 / 64
    X = torch.full((1, 8), 4.2e37, dtype=torch.bfloat16, device="cuda")  # h near the largest float
    f = hmoe.moe_few(p, X, top_k=1, act="relu")
    h = 8 * float(X[0, 0])
    assert np.isfinite(h) and np.abs(np64(f["Y"]) / (h / 8) - 1).max() <= 2.0 ** -8


def test_the_gater_of_kmeans():
    """R = C, r_bias = -|C|^2 / 2, one expert: Eq. 2's assignment and the training path's experts."""
    c_ = W.CONFIGS["tiny"]
    n, K = 60, c_.K
    inp = W.tiny_inputs(device="cuda", seed=1, n=n, bias=True)
    X, p = inp["X"], inp["params"]
    C = hmoe.kmeans_fit(X, K, 3, init_uniforms=inp["u"])["C"]
    a, _ = hmoe.kmeans_assign(X, C)
    few = dict(p, R=C, r_bias=-0.5 * C.double().pow(2).sum(1).float())
    f = hmoe.moe_few(few, X)
    assert torch.equal(f["expert"][:, 0], a) and bool((f["weight"] == 1).all())
    d = hmoe.moe_dispatch(a, K, rows=X)
    H = hmoe.moe_forward(p, d["rows_sorted"], d["offsets"], d["perm"], torch.tensor(inp["row_ptr"]).cuda(),
                         torch.tensor(inp["tag"]).cuda())["H"]
    assert (f["Y"] - H).abs().max() <= 1e-5 * H.abs().max()


def test_experts_past_32_bits():
    K, d, h, o = 66, 2048, 16384, 8  # 2.2e9 elements of W1
    p = {"R": torch.zeros(K, d, dtype=torch.bfloat16, device="cuda"), "r_bias": torch.zeros(K, device="cuda"),
         "W1": torch.empty(K, h, d, dtype=torch.bfloat16, device="cuda"), "b1": None, "b2": None,
         "W2": torch.empty(K, o, h, dtype=torch.bfloat16, device="cuda")}
    q = params(1, d, h, o, "bf16", "relu", False, 1)
    for k in ("W1", "W2"):
        p[k][K - 1] = q[k][0]
    p["r_bias"][K - 1] = 1.0
    X = torch.randn(2, d, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    f = hmoe.moe_few(p, X)
    assert (npi(f["expert"]) == K - 1).all()
    q["r_bias"] = None
    ref = hmoe.moe_few(q, X)
    assert torch.equal(f["Y"], ref["Y"])
    check(q, X, 1, "relu")


def test_streams_workspace_and_graphs():
    n, k = 11, 2
    p = params(20, 264, 136, 72, "bf16", "silu", True, 11)
    X = draw(p, n, k, "bf16", 12)
    prm = hmoe.make_few_params(p, k, "silu")
    a = hmoe.moe_few(p, X, top_k=k, act="silu")
    torch.cuda.synchronize()
    ws = torch.full((hmoe.moe_few_workspace(prm, n),), 255, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = hmoe.moe_few(prm, X, ws=ws)
        b2 = hmoe.moe_few(prm, X, ws=ws)  # the workspace as the first call left it
    s.synchronize()
    for key in a:
        assert torch.equal(a[key], b[key]) and torch.equal(a[key], b2[key]), key
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.moe_few(prm, X, ws=ws[:64])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hmoe.moe_few(prm, X, out=b, ws=ws)
    for seed in range(3):
        X.copy_(draw(p, n, k, "bf16", 20 + seed))
        ref = hmoe.moe_few(prm, X)
        for v in b.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for key in ref:
            assert torch.equal(b[key], ref[key]), key


def test_no_samples():
    p = params(4, 16, 8, 8, "bf16", "relu", False, 1)
    assert hmoe.moe_few(p, torch.empty(0, 16, dtype=torch.bfloat16, device="cuda"))["Y"].shape == (0, 8)


@pytest.mark.parametrize("dtype,n,K,d,h,o,k,act,bias", [
    # a sample's weights just below and above what one workgroup takes (224 KB)
    ("bf16", 7, 16, 224, 256, 208, 1, "relu", True), ("bf16", 7, 16, 224, 256, 216, 1, "relu", True),
    ("f32", 6, 3, 72, 104, 328, 3, "silu", False), ("f32", 6, 3, 72, 104, 144, 3, "silu", False),
    # few experts and rows of one vector, or of many
    ("bf16", 64, 500, 8, 24, 16, 8, "silu", True), ("f32", 3, 40, 8, 1000, 8, 2, "relu", True),
    ("bf16", 4, 2, 5000, 8, 2000, 1, "relu", True), ("bf16", 4, 2, 8, 5000, 8, 1, "silu", True)])
def test_layers_of_one_workgroup_a_sample(dtype, n, K, d, h, o, k, act, bias):
    p = params(K, d, h, o, dtype, act, bias, K + d)
    check(p, draw(p, n, k, dtype, n + h), k, act)


@pytest.mark.parametrize("K,d,h,o", [(4, 16, 24, 5000 * 8), (4, 32, 520, 264)])
@pytest.mark.parametrize("k", [1, 2])
def test_small_routers_before_large_experts(K, d, h, o, k):
    p = params(K, d, h, o, "bf16", "relu", True, K + d)
    p["r_bias"][1] = float("-inf")
    check(p, draw(p, 21, min(k, 2), "bf16", 5), k, "relu")
