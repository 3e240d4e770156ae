"""Low-rank adapters beside a shared projection, forward and backward, against a plain evaluation in 64 bits.

Tolerances (u = 2^-24).  A sum of N fp32 products in chains of at most N / 4 + 32 additions (an fp32 matrix
instruction takes 4 of K, then the joins) is off by at most c(N) = (N / 4 + 32) u times the sum of the terms'
absolute values.  U = s A x: c(d), and 2^-16 of itself for the two bf16 numbers that hold it; V = s B^T dY the
same with c(o).  Y, dX, dA and dB pass those on through the absolute values of what multiplies them and
add their own c().  bf16 outputs are rounded once: 2^-8 relative covers half an ulp."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64, npi

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def c(N):
    return (N / 4 + 32) * 2.0 ** -24


def adapters(E, d, o, r, dtype, bias, seed, scale=True):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s, std: (torch.randn(*s, generator=g) * std).to(DT[dtype]).cuda()
    return {"W": f(o, d, std=d ** -0.5), "b": f(o, std=0.3) if bias else None, "A": f(E, r, d, std=d ** -0.5),
            "B": f(E, o, r, std=r ** -0.5), "scale": (torch.rand(E, generator=g) + 0.5).cuda() if scale else None}


def rows(n, w, dtype, seed):
    return torch.randn(n, w, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).cuda()


def order(ids, E):
    """offsets and perm as the dispatch gives them, rows without an adapter last."""
    key = np.where((ids < 0) | (ids >= E), E, ids)
    off = np.zeros(E + 1, np.int32)
    off[1:] = np.cumsum(np.bincount(key, minlength=E + 1)[:E])
    return torch.tensor(off).cuda(), torch.tensor(np.argsort(key, kind="stable").astype(np.int32)).cuda()


def plain(p, X, ids, dY=None):
    """name -> (value, tolerance) in sample order."""
    x, W, A, B = (np64(t) for t in (X, p["W"], p["A"], p["B"]))
    E, r, d = A.shape
    o = W.shape[0]
    bf = X.dtype == torch.bfloat16
    split = 2.0 ** -16 if bf else 0.0
    b = np64(p["b"]) if p["b"] is not None else np.zeros(o)
    sc = np64(p["scale"]) if p["scale"] is not None else np.ones(E)
    Y = x @ W.T + b
    tY = c(d) * (np.abs(x) @ np.abs(W).T + np.abs(b))
    out = {}
    if dY is not None:
        dy = np64(dY)
        dX = dy @ W
        tX = c(o) * (np.abs(dy) @ np.abs(W))
        dA, tA, dB, tB = np.zeros(A.shape), np.zeros(A.shape), np.zeros(B.shape), np.zeros(B.shape)
    for e in range(E):
        i = np.nonzero(ids == e)[0]
        if not len(i):
            continue
        u = sc[e] * (x[i] @ A[e].T)
        eu = sc[e] * c(d) * (np.abs(x[i]) @ np.abs(A[e]).T) + split * np.abs(u)
        Y[i] += u @ B[e].T
        tY[i] += eu @ np.abs(B[e]).T + c(2 * r) * (np.abs(u) @ np.abs(B[e]).T)
        if dY is not None:
            v = sc[e] * (dy[i] @ B[e])
            ev = sc[e] * c(o) * (np.abs(dy[i]) @ np.abs(B[e])) + split * np.abs(v)
            dX[i] += v @ A[e]
            tX[i] += ev @ np.abs(A[e]) + c(2 * r) * (np.abs(v) @ np.abs(A[e]))
            N = min(len(i), 1024) + len(i) / 1024 * 4
            dB[e] = dy[i].T @ u
            tB[e] = np.abs(dy[i]).T @ (eu + c(N) * np.abs(u))
            dA[e] = v.T @ x[i]
            tA[e] = (ev + c(N) * np.abs(v)).T @ np.abs(x[i])
    out_round = 2.0 ** -8 if bf else 2.0 ** -23
    out["Y"] = (Y, tY + out_round * np.abs(Y))
    if dY is not None:
        out["dX"] = (dX, tX + out_round * np.abs(dX))
        out["dA"], out["dB"] = (dA, tA + 2.0 ** -23 * np.abs(dA)), (dB, tB + 2.0 ** -23 * np.abs(dB))
    return out


def close(got, ref, what, at=slice(None)):
    value, tol = ref
    off = ~(np.abs(np64(got)[at] - value[at]) <= tol[at])
    assert not off.any(), (what, off.sum(), np.argwhere(off)[:4], np64(got)[at][off][:4], value[at][off][:4],
                           tol[at][off][:4])


def ids_of(n, E, seed, none=0.1):
    rs = np.random.default_rng(seed)
    ids = rs.permutation(E)[np.minimum((E * rs.random(n) ** 2).astype(np.int64), E - 1)].astype(np.int32)
    ids[rs.random(n) < none] = -1
    return ids


def grouped(p, X, ids, dY, with_perm=True):
    """forward and backward of rows in sample order."""
    E = p["A"].shape[0]
    off, perm = order(ids, E)
    Xs = X[perm.long()].contiguous()
    f = hmoe.lora_forward(p, Xs, off, perm if with_perm else None)
    dYs = dY if with_perm else dY[perm.long()].contiguous()
    g = hmoe.lora_backward(p, Xs, off, dYs, f["U"], perm if with_perm else None)
    torch.cuda.synchronize()
    Y, dX = f["Y"], g["dX"]
    if not with_perm:
        back = torch.empty_like(perm.long())
        back[perm.long()] = torch.arange(len(ids), device="cuda")
        Y, dX = Y[back], dX[back]
    return {"Y": Y, "dX": dX, "dA": g["dA"], "dB": g["dB"]}


@pytest.mark.parametrize("dtype,n,E,d,o,r,bias", [
    ("f32", 1, 1, 8, 8, 8, False), ("bf16", 1, 3, 8, 16, 8, True), ("bf16", 7, 4, 72, 40, 24, True),
    ("f32", 16, 5, 64, 1000, 8, True), ("bf16", 17, 9, 200, 136, 16, False), ("bf16", 33, 33, 520, 264, 40, True),
    ("f32", 48, 7, 96, 104, 128, False), ("bf16", 64, 64, 1024, 2056, 32, True), ("bf16", 64, 1, 136, 72, 128, False),
    ("bf16", 5, 4096, 64, 88, 8, True), ("bf16", 48, 16, 256, 20000, 32, True), ("f32", 20, 3, 40, 16392, 16, False)])
def test_few_rows(dtype, n, E, d, o, r, bias):
    p = adapters(E, d, o, r, dtype, bias, n + o, scale=n % 2 == 0)
    X, ids = rows(n, d, dtype, n), ids_of(n, E, o)
    if n > 4:
        ids[2], ids[3] = E, 2 ** 31 - 1  # ids past the adapters: none
    Y = hmoe.lora_few(p, X, torch.tensor(ids).cuda())
    close(Y, plain(p, X, ids)["Y"], "Y")


@pytest.mark.parametrize("dtype,n,E,d,o,r", [
    # a wave's adapters take more loads than go out together, or fewer; wide outputs and narrow ones
    ("bf16", 64, 64, 64, 16392, 128), ("bf16", 64, 80, 72, 16400, 40), ("bf16", 33, 64, 136, 72, 104),
    ("bf16", 48, 16, 72, 16392, 72), ("bf16", 19, 30, 64, 16384, 8), ("f32", 50, 64, 72, 40, 72),
    ("f32", 64, 100, 64, 16392, 24), ("f32", 17, 2, 64, 136, 48)])
def test_loads_of_several_adapters(dtype, n, E, d, o, r):
    p = adapters(E, d, o, r, dtype, True, n + r, scale=True)
    X, ids = rows(n, d, dtype, n), np.random.default_rng(r).permutation(max(n, E))[:n].astype(np.int32) % E
    ids[1] = -1
    close(hmoe.lora_few(p, X, torch.tensor(ids).cuda()), plain(p, X, ids)["Y"], "Y")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,E", [(63, 1), (64, 1), (65, 1), (129, 2), (257, 1), (700, 3)])
def test_pieces_of_small_problems(dtype, n, E):
    """Adapters whose rows end at, before and past a piece of the smallest size."""
    d, o, r = 72, 88, 16
    p = adapters(E, d, o, r, dtype, False, n)
    X, dY, ids = rows(n, d, dtype, n), rows(n, o, dtype, n + 1), np.sort(np.arange(n) % (E + 1) % E).astype(np.int32)
    got, ref = grouped(p, X, ids, dY), plain(p, X, ids, dY)
    for k in ("dA", "dB"):
        close(got[k], ref[k], k)


@pytest.mark.parametrize("dtype,n,E,d,o,r,bias", [
    ("f32", 1, 1, 8, 8, 8, True), ("bf16", 2, 3, 16, 8, 8, False), ("bf16", 300, 5, 72, 136, 24, True),
    ("f32", 777, 8, 64, 1000, 8, True), ("bf16", 1000, 300, 64, 104, 16, False), ("bf16", 2500, 3, 136, 72, 128, True),
    ("f32", 2100, 2, 40, 56, 72, False), ("bf16", 3000, 40, 2048, 2048, 64, True), ("bf16", 5000, 128, 264, 4104, 16, True),
    ("f32", 1500, 100, 520, 2048, 40, True), ("bf16", 4099, 1, 1024, 1024, 32, False)])
@pytest.mark.parametrize("with_perm", [True, False])
def test_many_rows_and_gradients(dtype, n, E, d, o, r, bias, with_perm):
    p = adapters(E, d, o, r, dtype, bias, n + o, scale=n % 2 == 0)
    X, dY, ids = rows(n, d, dtype, n), rows(n, o, dtype, n + 1), ids_of(n, E, n)
    got, ref = grouped(p, X, ids, dY, with_perm), plain(p, X, ids, dY)
    for k in ("Y", "dX", "dA", "dB"):
        close(got[k], ref[k], k)


@pytest.mark.parametrize("dtype,d,o,r", [("bf16", 264, 136, 24), ("f32", 72, 200, 16), ("bf16", 136, 72, 40),
                                          ("bf16", 2056, 1032, 16), ("f32", 520, 88, 32)])
@pytest.mark.parametrize("adapter", [2, -1, 5])
def test_one_row(dtype, d, o, r, adapter):
    """Formed in one launch (narrow adapters) and in two, with and without an adapter."""
    p = adapters(5, d, o, r, dtype, True, d)
    X, ids = rows(1, d, dtype, o), np.array([adapter], np.int32)
    close(hmoe.lora_few(p, X, torch.tensor(ids).cuda()), plain(p, X, ids)["Y"], "Y")


@pytest.mark.parametrize("dtype,n,E,d,o,r", [
    ("bf16", 16500, 9, 1032, 136, 24),  # whole tiles that gather dY's rows
    ("bf16", 9000, 5, 264, 2312, 40),   # whole tiles forward
    ("bf16", 200, 3, 1032, 72, 24),     # reductions split among workgroups
    ("f32", 130, 4, 72, 1032, 8), ("bf16", 17000, 3, 40, 72, 48)])  # adapters of many pieces
def test_tilings(dtype, n, E, d, o, r):
    p = adapters(E, d, o, r, dtype, True, n + o)
    X, dY, ids = rows(n, d, dtype, n), rows(n, o, dtype, n + 1), ids_of(n, E, n)
    got, ref = grouped(p, X, ids, dY), plain(p, X, ids, dY)
    for k in ("Y", "dX", "dA", "dB"):
        close(got[k], ref[k], k)


@pytest.mark.parametrize("dtype,n,E,d,o,r", [
    # a workgroup of eight waves or of four to 16 columns, few and many of them, groups short of the waves
    ("bf16", 1, 3, 2040, 4096, 16), ("bf16", 1, 3, 2048, 4104, 16), ("f32", 1, 3, 1032, 72, 24), ("bf16", 1, 3, 4104, 88, 32),
    ("bf16", 24, 30, 72, 4096, 24), ("bf16", 40, 7, 264, 6008, 16), ("f32", 64, 20, 136, 4104, 40),
    ("bf16", 64, 20, 1032, 1000, 128)])
def test_waves_of_a_workgroup(dtype, n, E, d, o, r):
    p = adapters(E, d, o, r, dtype, True, n + o, scale=True)
    X, ids = rows(n, d, dtype, n), ids_of(n, E, o)
    if n == 1:
        ids[0] = 1
    close(hmoe.lora_few(p, X, torch.tensor(ids).cuda()), plain(p, X, ids)["Y"], "Y")


@pytest.mark.parametrize("dtype,n,E,d,o,r", [
    # gradients: ranks that take one chunk of U or several, tiles of 64 and of 256 columns, long adapters
    ("bf16", 1200, 70, 520, 1032, 16), ("bf16", 1200, 70, 520, 1032, 104), ("f32", 1200, 70, 520, 264, 32),
    ("f32", 900, 70, 264, 1032, 72), ("bf16", 6000, 2, 136, 264, 88)])
def test_chunks_of_the_rank(dtype, n, E, d, o, r):
    p = adapters(E, d, o, r, dtype, False, n + o)
    X, dY, ids = rows(n, d, dtype, n), rows(n, o, dtype, n + 1), ids_of(n, E, n)
    got, ref = grouped(p, X, ids, dY), plain(p, X, ids, dY)
    for k in ("dA", "dB"):
        close(got[k], ref[k], k)


@pytest.mark.parametrize("dtype,n,E,d,o,r", [
    ("bf16", 8000, 5, 1032, 136, 16),  # whole tiles on half of the chip, gathering
    ("bf16", 4700, 3, 200, 616, 8), ("f32", 4700, 3, 200, 616, 8)])  # reductions in three splits
def test_half_filled_tilings(dtype, n, E, d, o, r):
    p = adapters(E, d, o, r, dtype, True, n + o)
    X, dY, ids = rows(n, d, dtype, n), rows(n, o, dtype, n + 1), ids_of(n, E, n)
    got, ref = grouped(p, X, ids, dY), plain(p, X, ids, dY)
    for k in ("Y", "dX", "dA", "dB"):
        close(got[k], ref[k], k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_adapters_and_adapters_without_rows(dtype):
    n, E, d, o, r = 600, 6, 72, 88, 16
    p = adapters(E, d, o, r, dtype, True, 1)
    X, dY = rows(n, d, dtype, 2), rows(n, o, dtype, 3)
    for ids in (np.full(n, -1, np.int32), np.full(n, 4, np.int32), np.repeat([0, 5], n // 2).astype(np.int32)):
        got, ref = grouped(p, X, ids, dY), plain(p, X, ids, dY)
        for k in got:
            close(got[k], ref[k], k)
        for e in range(E):
            if not (ids == e).any():
                assert (got["dA"][e] == 0).all() and (got["dB"][e] == 0).all()


def test_a_bad_row_stays_alone():
    """NaN in a row, and in an adapter that one row has: no other row sees it."""
    n, E, d, o, r = 50, 4, 72, 88, 16
    p = adapters(E, d, o, r, "bf16", True, 4)
    X, ids = rows(n, d, "bf16", 5), np.arange(n).astype(np.int32) % 3
    ids[20] = 3
    X[11, 3] = float("nan")
    p["A"][3] = float("nan")
    p["B"][3] = float("inf")
    keep = np.ones(n, bool)
    keep[[11, 20]] = False
    clean = X.clone()
    clean[11] = 0
    safe = dict(p, A=p["A"].clone(), B=p["B"].clone())
    safe["A"][3], safe["B"][3] = 0, 0
    ref = plain(safe, clean, ids)["Y"]
    Y = hmoe.lora_few(p, X, torch.tensor(ids).cuda())
    close(Y, ref, "few", keep)
    off, perm = order(ids, E)
    f = hmoe.lora_forward(p, X[perm.long()].contiguous(), off, perm)
    close(f["Y"], ref, "many", keep)
    assert np.isnan(np64(Y)[[11, 20]]).all() and np.isnan(np64(f["Y"])[[11, 20]]).all()


def test_both_forms_agree():
    n, E, d, o, r = 64, 9, 512, 1024, 32
    p = adapters(E, d, o, r, "bf16", True, 6)
    X, ids = rows(n, d, "bf16", 7), ids_of(n, E, 8)
    off, perm = order(ids, E)
    a = hmoe.lora_few(p, X, torch.tensor(ids).cuda())
    b = hmoe.lora_forward(p, X[perm.long()].contiguous(), off, perm)["Y"]
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * a.float().abs().max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_against_differences(dtype):
    """<dA, E>, <dB, E> and <dX, E> against central differences of the 64-bit forward's <dY, Y>, which is
    linear in each: exact but for 64-bit rounding.  The gradients' own tolerance, summed against |E|."""
    n, E, d, o, r = 90, 4, 40, 56, 8
    p = adapters(E, d, o, r, dtype, True, 9)
    X, dY, ids = rows(n, d, dtype, 10), rows(n, o, dtype, 11), ids_of(n, E, 12)
    got, ref = grouped(p, X, ids, dY), plain(p, X, ids, dY)
    rs = np.random.default_rng(13)
    sc, b, W = np64(p["scale"]), np64(p["b"]), np64(p["W"])

    def value(x, A, B):
        Y = x @ W.T + b
        for i in range(n):
            if ids[i] >= 0:
                Y[i] += sc[ids[i]] * (B[ids[i]] @ (A[ids[i]] @ x[i]))
        return (np64(dY) * Y).sum()

    at = {"dX": np64(X), "dA": np64(p["A"]), "dB": np64(p["B"])}
    for k in at:
        D = rs.standard_normal(at[k].shape)
        up, dn = dict(at), dict(at)
        up[k], dn[k] = at[k] + D, at[k] - D
        diff = (value(up["dX"], up["dA"], up["dB"]) - value(dn["dX"], dn["dA"], dn["dB"])) / 2
        assert abs((np64(got[k]) * D).sum() - diff) <= (ref[k][1] * np.abs(D)).sum() + 1e-9 * abs(diff), k


def test_gradients_one_at_a_time():
    n, E, d, o, r = 500, 4, 72, 88, 16
    p = adapters(E, d, o, r, "bf16", False, 14)
    X, dY, ids = rows(n, d, "bf16", 15), rows(n, o, "bf16", 16), ids_of(n, E, 17)
    off, perm = order(ids, E)
    Xs = X[perm.long()].contiguous()
    f = hmoe.lora_forward(p, Xs, off, perm)
    g = hmoe.lora_backward(p, Xs, off, dY, f["U"], perm)
    only = hmoe.lora_backward(p, Xs, off, dY, f["U"], perm, want_adapters=False)
    assert only["dA"] is None and torch.equal(only["dX"], g["dX"])
    only = hmoe.lora_backward(p, Xs, off, dY, f["U"], perm, want_dX=False)
    assert only["dX"] is None and torch.equal(only["dA"], g["dA"]) and torch.equal(only["dB"], g["dB"])


def test_output_past_32_bits():
    n, E, d, o, r = 70000, 2, 8, 32768, 8  # 2.3e9 outputs
    p = adapters(E, d, o, r, "bf16", True, 18)
    X = rows(n, d, "bf16", 19)
    ids = (np.arange(n) % 3 - 1).astype(np.int32)
    off, perm = order(ids, E)
    f = hmoe.lora_forward(p, X[perm.long()].contiguous(), off, perm)
    at = np.array([0, 1, 2, 35000, 65535, 65536, 69997, 69998, 69999])
    ref = plain(p, X[torch.tensor(at)], ids[at])["Y"]
    close(f["Y"][torch.tensor(at).cuda()], ref, "Y")
    dY = torch.zeros(n, o, dtype=torch.bfloat16, device="cuda")
    dY[torch.tensor(at).cuda()] = rows(len(at), o, "bf16", 20)
    g = hmoe.lora_backward(p, X[perm.long()].contiguous(), off, dY, f["U"], perm)
    want = plain(p, X[torch.tensor(at)], ids[at], dY[torch.tensor(at).cuda()])
    close(g["dX"][torch.tensor(at).cuda()], want["dX"], "dX")
    for k in ("dA", "dB"):
        close(g[k], want[k], k)


def test_streams_workspaces_and_graphs():
    n, E, d, o, r = 1300, 5, 136, 264, 24
    p = adapters(E, d, o, r, "bf16", True, 21)
    prm = hmoe.make_lora(p)
    X, dY, ids = rows(n, d, "bf16", 22), rows(n, o, "bf16", 23), ids_of(n, E, 24)
    few_ids = torch.tensor(ids[:40]).cuda()
    off, perm = order(ids, E)
    Xs = X[perm.long()].contiguous()
    ws = torch.full((hmoe.lora_workspace(prm, n),), 255, dtype=torch.uint8, device="cuda")
    wf = torch.full((hmoe.lora_few_workspace(prm, 40),), 255, dtype=torch.uint8, device="cuda")

    def step(out):
        f = hmoe.lora_forward(prm, Xs, off, perm, out=out, ws=ws)
        g = hmoe.lora_backward(prm, Xs, off, dY, f["U"], perm, out=out, ws=ws)
        y = hmoe.lora_few(prm, X[:40], few_ids, out=out.get("few"), ws=wf)
        return {"Y": f["Y"], "U": f["U"], "dX": g["dX"], "dA": g["dA"], "dB": g["dB"], "few": y}

    a = step({})
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = step({})
    s.synchronize()
    for k in a:
        if k != "U":  # rows without an adapter have nothing there
            assert torch.equal(a[k], b[k]), k
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.lora_forward(prm, Xs, off, perm, ws=ws[:64])
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.lora_few(prm, X[:40], few_ids, ws=wf[:64])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    for seed in range(3):
        X.copy_(rows(n, d, "bf16", 30 + seed))
        Xs.copy_(X[perm.long()])
        ref = {k: v.clone() for k, v in step(a).items()}
        for v in b.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            if k != "U":
                assert torch.equal(b[k], ref[k]), k


def test_no_rows():
    p = adapters(3, 16, 24, 8, "bf16", True, 1)
    e = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert hmoe.lora_few(p, e, torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 24)
    f = hmoe.lora_forward(p, e, off)
    g = hmoe.lora_backward(p, e, off, f["Y"], f["U"])
    assert f["Y"].shape == (0, 24) and (g["dA"] == 0).all() and (g["dB"] == 0).all()
