"""Token log-probabilities, entropies, alternatives and their gradient against a plain evaluation in
64 bits.

Tolerances (u = 2^-24).  A term e^(s d), d = x - max: s d carries three roundings of relative size u
(the difference, the scale times log2 e, the product), 3 u |s d| of the term, at most 3 u / e of the
largest; v_exp_f32 and the sums' roundings add some u for each of up to a few hundred additions, which
are of either sign: ln S is taken to 1e-5.  logp = s d - ln S: 1e-5 + 4 u |logp|.  The entropy adds the
quotient s T / S <= ln V, with the same relative error: 1e-5 (1 + ln V).  The gradient's terms carry
e^(ln p) with the error of ln p, 1e-5 + 4 u |ln p| <= 5e-5 down to p = 2^-126 (below it p is 0: 2^-125 of
the gradients): 1e-4 of the terms' absolute sum, and for bf16 the output's rounding, 2^-8 of the value
(half an ulp is 2^-9).  Indexes are exact."""
import math

import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from paper_1704_06363_amd import workloads as W
from tests.parity import anchor_of_columns, np64, npi

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


def plain(x, scale, token, m):
    """logp, entropy, lse, top_idx, top_logp of rows x (float64)."""
    n, V = x.shape
    with np.errstate(all="ignore"):
        mx = np.max(np.where(np.isnan(x), -INF, x), axis=1)
        empty = ~np.isnan(x).any(1) & (mx == -INF)
        d = scale * (x - np.where(empty, 0.0, mx)[:, None])
        e = np.exp(d)
        S = e.sum(1)
        ls = np.where(empty, -INF, np.log(S))
        lp = d - np.where(empty, 0.0, ls)[:, None]
        p = np.exp(lp)
        ent = np.where(empty, 0.0, -np.where(p == 0, 0.0, p * lp).sum(1))
        lse = np.where(empty, -INF, scale * mx + ls)
        bad = np.isnan(x).any(1) | (mx == INF)
        lp[bad] = np.nan
        ent[bad] = np.nan
        lse[bad] = np.nan
    ok = (token >= 0) & (token < V)
    logp = np.where(ok, lp[np.arange(n), np.where(ok, token, 0)], 0.0)
    # value descending, index ascending, NaN last
    order = np.lexsort((np.broadcast_to(np.arange(V), x.shape), -np.where(np.isnan(x), -INF, x), np.isnan(x)), axis=1)
    idx = order[:, :m]
    return logp, ent, lse, idx, np.take_along_axis(lp, idx, 1), lp


def plain_grad(lp, ent, scale, token, gl, ge):
    n, V = lp.shape
    with np.errstate(all="ignore"):
        p = np.exp(lp)
        plp = np.where(p == 0, 0.0, p * lp)
    p = np.where(np.isnan(p), np.nan, p)
    hot = np.zeros((n, V))
    ok = (token >= 0) & (token < V)
    hot[np.nonzero(ok)[0], token[ok]] = 1.0
    glk = np.where(ok, gl, 0.0)[:, None]
    gek = ge[:, None]
    empty = (lp == -INF).all(1)  # nothing to move: 0 by definition
    hot[empty] = 0.0
    g = scale * (glk * (hot - p) - gek * (plp + p * ent[:, None]))
    size = scale * (np.abs(glk) * (hot + p) + np.abs(gek) * (np.abs(plp) + p * np.abs(ent[:, None])))
    return g, size


def close(got, ref, tol, what):
    got = np64(got)
    assert got.shape == ref.shape, what
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))
    with np.errstate(all="ignore"):
        off = ~same & ~(np.abs(got - ref) <= tol)
    assert not off.any(), (what, np.argwhere(off)[:4], got[off][:4], ref[off][:4])


def check(logits, token, m, scale, anchor=None, full=None):
    x = np64(logits) if full is None else full
    n, V = x.shape
    t = npi(token)
    logp, ent, lse, idx, tlp, lp = plain(x, scale, t, m)
    f = hmoe.token_logprob(logits, token, m=m, scale=scale, anchor=anchor)
    torch.cuda.synchronize()
    u = 2.0 ** -24
    close(f["logp"], logp, 1e-5 + 4 * u * np.abs(logp), "logp")
    close(f["entropy"], ent, 1e-5 * (1 + math.log(V)), "entropy")
    with np.errstate(all="ignore"):
        close(f["lse"], lse, 1e-5 + 4 * u * np.abs(lse), "lse")
    if m:
        assert np.array_equal(npi(f["top_idx"]), idx)
        close(f["top_logp"], tlp, 1e-5 + 4 * u * np.where(np.isfinite(tlp), np.abs(tlp), 0), "top_logp")
    return f, lp, ent


def check_grad(logits, token, scale, f, lp, ent, seed, anchor=None, in_place=False, ld=None):
    n, V = lp.shape
    rs = np.random.default_rng(seed)
    gl, ge = rs.standard_normal(n).astype(np.float32), rs.standard_normal(n).astype(np.float32)
    G = lambda a: torch.tensor(a, device="cuda")
    ref, size = plain_grad(lp, ent, scale, npi(token), gl.astype(np.float64), ge.astype(np.float64))
    out = None
    if ld:
        out = torch.full((n, ld), 7.0, dtype=logits.dtype, device="cuda")[:, :V]
    if in_place:
        logits = logits.clone() if logits.is_contiguous() else logits
        out = logits
    got = hmoe.token_logprob_backward(logits, token, f["stat"], f["entropy"], G(gl), G(ge), scale=scale, anchor=anchor,
                                      out=out)
    torch.cuda.synchronize()
    tol = 1e-4 * size + 2.0 ** -124
    if logits.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(ref)
    close(got, ref, tol, "dlogits")
    if ld and ld > V:
        assert bool((got.as_strided((n, ld - V), (ld, 1), V) == 7.0).all())  # nothing behind the rows


def rows(n, V, pad, dtype, seed, ties=False, std=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-8, 9, (n, V + pad), generator=g).float() if ties else torch.randn(n, V + pad, generator=g) * std
    x = x.to(DT[dtype]).cuda()
    if pad:
        x[:, V:] = float("nan")
    return x[:, :V]


def tokens(n, V, seed):
    return torch.tensor(np.random.default_rng(seed).integers(0, V, n).astype(np.int32), device="cuda")


@pytest.mark.parametrize("dtype,n,V,pad,m,scale,ties", [
    ("bf16", 1, 1, 0, 1, 1.0, False), ("f32", 3, 7, 1, 7, 0.5, False), ("bf16", 5, 8, 0, 8, 1.0, True),
    ("f32", 2, 3, 0, 0, 2.0, False), ("bf16", 4, 13, 3, 13, 1.0, True), ("bf16", 2, 100003, 0, 16, 1 / 0.7, False),
    ("f32", 1, 50021, 5, 16, 1.0, False), ("bf16", 1501, 1000, 0, 10, 1.0, False),
    ("bf16", 1025, 1001, 8, 3, 1.0, True), ("f32", 1030, 2051, 1, 5, 0.9, False), ("f32", 1024, 8192, 0, 1, 1.0, True),
    ("bf16", 530, 8193, 0, 16, 1.0, True), ("bf16", 33, 50000, 0, 0, 1.0, False), ("bf16", 9, 50000, 0, 16, 1.0, True),
    ("f32", 64, 4097, 3, 2, 1.3, False), ("bf16", 513, 16000, 0, 4, 1.0, False)])
def test_rows_of_any_size(dtype, n, V, pad, m, scale, ties):
    x, t = rows(n, V, pad, dtype, n + V, ties), tokens(n, V, n)
    f, lp, ent = check(x, t, m, scale)
    check_grad(x, t, scale, f, lp, ent, V, ld=V + 2 * pad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(14, 300), (14, 20000), (1400, 517)])  # a wave, pieces of a row, many rows
def test_masked_infinite_and_missing_entries(dtype, n, V):
    x = rows(n, V, 0, dtype, 3).clone()
    low = torch.finfo(DT[dtype]).min
    for i in range(0, n, 14):
        x[i] = -INF                                   # nothing left
        x[i + 1] = -INF; x[i + 1, V // 2] = 1.5       # one entry
        x[i + 2] = -INF; x[i + 2, V - 5:] = 0.25      # fewer than the alternatives, at the end
        x[i + 3] = low                                # the lowest finite value everywhere
        x[i + 4, : V // 2] = low                      # and as a mask, before the other entries
        x[i + 5, V // 3:] = low                       # and behind them
        x[i + 6, 3] = float("nan")
        x[i + 7, V - 1] = INF
        x[i + 8] = float("nan")
        x[i + 9] = -INF; x[i + 9, 7] = float("nan")
        x[i + 10, ::2] = -INF
        x[i + 11] = x[i + 11] * 1000.0                # large logits
        x[i + 12] = 2.0                               # all equal
        x[i + 13, V // 2:] = torch.arange(V - V // 2, device="cuda").to(x.dtype)  # ascending
    t = tokens(n, V, 5)
    f, lp, ent = check(x, t, 9, 1.0)
    check_grad(x, t, 1.0, f, lp, ent, 1)
    check(x, t, 16, 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,m", [(3, 5, 5), (6, 700, 16), (4, 30000, 9), (1300, 300, 3)])
def test_zeros_of_either_sign_among_the_best(dtype, n, V, m):
    """Rows whose m-th entry is +0 or -0 (equal, by index), and rows of nothing above 0."""
    x = -rows(n, V, 0, dtype, 6).abs() - 0.5
    at = torch.randint(0, V, (n, 40), generator=torch.Generator().manual_seed(7)).cuda()
    x.scatter_(1, at[:, ::2], 0.0)
    x.scatter_(1, at[:, 1::2], -0.0)
    x[1::3, V // 2] = 1.0
    x[2] = 0.0
    f, lp, ent = check(x, tokens(n, V, 8), m, 1.0)
    check_grad(x, tokens(n, V, 8), 1.0, f, lp, ent, 9)


def test_rows_without_a_token():
    x, t = rows(40, 999, 0, "bf16", 1), tokens(40, 999, 1)
    t[::3] = -1
    t[1::7] = 999
    t[2] = 2 ** 31 - 1
    f, lp, ent = check(x, t, 2, 1.0)
    check_grad(x, t, 1.0, f, lp, ent, 2)
    only = hmoe.token_logprob(x, None, m=2)
    assert only["logp"] is None and torch.equal(only["entropy"], f["entropy"])
    assert torch.equal(only["top_idx"], f["top_idx"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_in_place_and_of_one_output(dtype):
    n, V = 21, 5003
    x, t = rows(n, V, 0, dtype, 4), tokens(n, V, 4)
    f, lp, ent = check(x, t, 0, 1.5)
    check_grad(x, t, 1.5, f, lp, ent, 3, in_place=True)
    g = torch.randn(n, device="cuda")
    both = [hmoe.token_logprob_backward(x, t, f["stat"], f["entropy"], g, torch.zeros_like(g), scale=1.5),
            hmoe.token_logprob_backward(x, t, f["stat"], None, g, None, scale=1.5)]
    assert torch.equal(both[0], both[1])
    both = [hmoe.token_logprob_backward(x, t, f["stat"], f["entropy"], torch.zeros_like(g), g, scale=1.5),
            hmoe.token_logprob_backward(x, None, f["stat"], f["entropy"], None, g, scale=1.5)]
    assert torch.equal(both[0], both[1])


def test_gradient_against_differences():
    """Central differences of the 64-bit values with a step h: their error is h^2 times a third
    derivative of a few units (1e-8), and the kernel's fp32 gradient is good to 1e-4 of its terms."""
    n, V, scale, h = 3, 37, 0.8, 1e-4
    x, t = rows(n, V, 0, "f32", 8, std=1.0), tokens(n, V, 8)
    f = hmoe.token_logprob(x, t, scale=scale)
    gl, ge = torch.tensor([0.7, -1.2, 0.4], device="cuda"), torch.tensor([0.3, 0.9, -1.1], device="cuda")
    got = np64(hmoe.token_logprob_backward(x, t, f["stat"], f["entropy"], gl, ge, scale=scale))
    x0, tk = np64(x), npi(t)
    value = lambda y: plain(y, scale, tk, 0)
    for v in range(V):
        up, dn = x0.copy(), x0.copy()
        up[:, v] += h
        dn[:, v] -= h
        a, b = value(up), value(dn)
        diff = (np64(gl) * (a[0] - b[0]) + np64(ge) * (a[1] - b[1])) / (2 * h)
        assert np.abs(got[:, v] - diff).max() <= 1e-4 * 4 + 1e-6


@pytest.mark.parametrize("dtype,n,V", [("bf16", 70, 1000), ("f32", 35, 520), ("bf16", 3, 20000)])
def test_logits_as_the_forward_stores_them(dtype, n, V):
    d, h, o, K = 64, 128, 64, 4
    p = W.moe_params(K, d, h, o, V, 5, dtype, "cuda", bias=True)
    X = W.rectified_gaussian(n, d, 6, dtype, "cuda") * 4
    r = hmoe.moe_dispatch(torch.arange(n, device="cuda", dtype=torch.int32) % K, K, rows=X)
    rp, tg = W.zipf_labels(n, V, 3, 7)
    f = hmoe.moe_forward(p, r["rows_sorted"], r["offsets"], r["perm"], torch.tensor(rp).cuda(), torch.tensor(tg).cuda(),
                         save_logits=True)
    a = anchor_of_columns(f["logit_anchor"], V)
    full = (a.astype(np.float32) + np64(f["logits"]).astype(np.float32)).astype(np.float64)
    t = tokens(n, V, 9)
    g, lp, ent = check(f["logits"], t, 12, 1.0, anchor=f["logit_anchor"], full=full)
    check_grad(f["logits"], t, 1.0, g, lp, ent, 4, anchor=f["logit_anchor"])
    top, val = hmoe.topm(f["logits"], 12, want_values=True, anchor=f["logit_anchor"])
    assert torch.equal(top, g["top_idx"])


def test_rows_further_apart_than_32_bits():
    n, V, ld = 3, 1003, (1 << 31) + 24
    flat = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((n, V), (ld, 1))
    x.copy_(rows(n, V, 0, "bf16", 2))
    t = tokens(n, V, 2)
    f, lp, ent = check(x, t, 4, 1.0)
    check_grad(x, t, 1.0, f, lp, ent, 6, in_place=True)


def test_more_rows_than_a_launch_takes():
    n, V = (1 << 24) + 9, 4
    x = torch.randn(n, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    t = torch.randint(0, V, (n,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda",
                      dtype=torch.int32)
    f = hmoe.token_logprob(x, t, m=1)
    lp = torch.log_softmax(x.double(), 1)
    assert (f["logp"] - lp.gather(1, t.long()[:, None])[:, 0]).abs().max() <= 1e-5 * 2
    first = torch.where(x == x.amax(1, keepdim=True), torch.arange(V, device="cuda"), V).amin(1)  # of equal ones
    assert torch.equal(f["top_idx"][:, 0].long(), first)
    g = hmoe.token_logprob_backward(x, t, f["stat"], None, torch.ones(n, device="cuda"))
    ref = -lp.exp()
    ref.scatter_add_(1, t.long()[:, None], torch.ones(n, 1, dtype=torch.float64, device="cuda"))
    assert (g - ref).abs().max() <= 1e-4


def test_streams_workspace_and_repeated_calls():
    n, V, m = 5, 30011, 16
    x, t = rows(n, V, 0, "bf16", 1), tokens(n, V, 1)
    a = hmoe.token_logprob(x, t, m=m)
    torch.cuda.synchronize()
    ws = torch.full((hmoe.token_logprob_workspace(n, V, m, torch.bfloat16),), 255, dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = hmoe.token_logprob(x, t, m=m, ws=ws)
    s.synchronize()
    for k in a:
        assert torch.equal(a[k], b[k]), k
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.token_logprob(x, t, m=m, ws=ws[:64])


def test_captured_in_a_graph():
    n, V, m = 6, 20011, 5
    x, t = rows(n, V, 0, "f32", 1), tokens(n, V, 1)
    g = torch.randn(n, device="cuda")
    out = {k: v for k, v in hmoe.token_logprob(x, t, m=m).items()}
    ws = torch.empty(hmoe.token_logprob_workspace(n, V, m, torch.float32), dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(x)

    def both():
        f = hmoe.token_logprob(x, t, m=m, out=out, ws=ws)
        hmoe.token_logprob_backward(x, t, f["stat"], f["entropy"], g, g, out=dx)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(3):
        x.copy_(rows(n, V, 0, "f32", 50 + seed))
        e = hmoe.token_logprob(x, t, m=m)
        ref = hmoe.token_logprob_backward(x, t, e["stat"], e["entropy"], g, g)
        for v in out.values():
            v.zero_()
        dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], e[k]), k
        assert torch.equal(dx, ref)


def test_no_rows():
    x = torch.empty(0, 100, dtype=torch.bfloat16, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    f = hmoe.token_logprob(x, t, m=3)
    assert f["top_idx"].shape == (0, 3)
    assert hmoe.token_logprob_backward(x, t, f["stat"], None, f["logp"]).shape == (0, 100)
