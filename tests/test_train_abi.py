"""The entry points of include/hmoe_train.h: exported, bound, and refusing bad arguments before anything is
launched (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

from paper_1704_06363_amd import hmoe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = ctypes.c_float
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hmoe.LIB_PATH):
        from paper_1704_06363_amd import build
        build.build()
    return hmoe.lib()


def refused(rc, code, word):
    assert rc == code and word in hmoe.last_error(), (rc, hmoe.last_error())


def test_exports_every_declared_symbol(lib):
    src = open(os.path.join(ROOT, "include", "hmoe_train.h")).read()
    names = sorted(set(re.findall(r"\b(hmoe_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", src, flags=re.S))))
    assert set(names) == set(hmoe.TRAIN_SYMBOLS)
    for name in names:
        assert hasattr(lib, name), name


def router(K=16, d=64, top_k=2, dt=1, renorm=0, R=16, bias=16):
    return hmoe.Router(K, d, top_k, dt, renorm, R, bias)


def test_router_refusals(lib):
    big = 1 << 40

    def call(p=None, n=10, X=16, expert=16, weight=16, scores=16, counts=16, share=16, loss=16, ws=16, wb=big, **kw):
        p = ctypes.byref(router(**kw)) if p is None else p
        return lib.hmoe_router_forward(p, n, X, expert, weight, scores, counts, share, loss, ws, wb, None)

    def both(word, code, **kw):
        refused(call(**kw), code, word)
        n = kw.pop("n", 10)
        refused(lib.hmoe_router_backward(ctypes.byref(router(**kw)), n, 16, 16, 16, 16, 16, F(0.1), F(0.1), 16, 16, 16, 16,
                                         big, None), code, word)
        assert lib.hmoe_router_workspace(ctypes.byref(router(**kw)), n) == 0

    both("dtype", -2, dt=7)
    both("K =", -1, K=0)
    both("K =", -1, K=4097)
    both("d =", -3, d=60)
    both("d =", -3, d=0)
    both("exceeds", -1, d=(1 << 20) + 8)
    for k in (0, -1, 9):
        both("top_k", -1, top_k=k)
    both("top_k", -1, K=3, top_k=4)
    both("n =", -1, n=-1)
    both("n =", -1, n=(1 << 28) + 1)
    refused(lib.hmoe_router_forward(None, 1, 16, 16, 16, 16, 16, 16, 16, 16, big, None), -1, "params")
    for key in ("X", "expert", "weight", "scores", "counts", "share", "loss"):
        refused(call(**{key: None}), -1, key)
    for key in ("X", "scores"):
        refused(call(**{key: 20}), -3, key)
    refused(call(R=None), -1, "R is NULL")
    refused(call(R=20), -3, "R is not")
    need = lib.hmoe_router_workspace(ctypes.byref(router()), 10)
    assert need > 0
    refused(call(wb=need - 1), -4, "workspace")
    refused(call(ws=None), -4, "workspace")
    refused(call(ws=24), -3, "workspace")

    def grad(n=10, X=16, scores=16, expert=16, counts=16, gw=16, balance=0.1, z=0.1, dX=16, dR=16, db=16, ws=16, wb=big, **kw):
        return lib.hmoe_router_backward(ctypes.byref(router(**kw)), n, X, scores, expert, counts, gw, F(balance), F(z), dX, dR,
                                        db, ws, wb, None)
    for bad in (NAN, INF):
        refused(grad(balance=bad), -1, "balance")
        refused(grad(z=bad), -1, "z =")
    for key in ("X", "scores", "expert", "counts"):
        refused(grad(**{key: None}), -1, key)
    for key in ("X", "scores", "dX", "dR"):
        refused(grad(**{key: 24}), -3, key)
    refused(grad(R=None), -1, "R is NULL")
    refused(grad(wb=16), -4, "workspace")
    assert grad(dX=None, dR=None, db=None) == 0  # nothing is wanted


def join(d=64, k=1, dt=1, norm=1, scale=1.0, eps=1e-6, gy=16, gh=16):
    return ctypes.byref(hmoe.Join(d, k, dt, norm, scale, eps, gy, gh))


def test_join_refusals(lib):
    big = 1 << 40

    def call(n=10, x=16, y=32, gate=16, xo=64, h=128, **kw):
        return lib.hmoe_join_forward(join(**kw), n, x, y, gate, xo, h, None)

    def grad(n=10, xo=16, y=32, gate=16, dxo=16, dh=16, dx=64, dy=128, dg=16, gy_=16, gh_=16, ws=16, wb=big, **kw):
        return lib.hmoe_join_backward(join(**kw), n, xo, y, gate, dxo, dh, dx, dy, dg, gy_, gh_, ws, wb, None)

    for word, code, kw in (("dtype", -2, dict(dt=5)), ("d =", -3, dict(d=12)), ("exceeds", -1, dict(d=32776)),
                           ("k =", -1, dict(k=9)), ("k =", -1, dict(k=-1)), ("scale", -1, dict(scale=NAN)),
                           ("scale", -1, dict(scale=INF)), ("eps", -1, dict(eps=0.0)), ("eps", -1, dict(eps=NAN)),
                           ("eps", -1, dict(eps=-1.0)), ("eps", -1, dict(eps=INF)), ("gamma_y", -3, dict(gy=24)),
                           ("gamma_h", -3, dict(gh=24)), ("n =", -1, dict(n=-1)), ("n =", -1, dict(n=1 << 31))):
        refused(call(**kw), code, word)
        refused(grad(**kw), code, word)
    refused(call(x=None), -1, "x is NULL")
    refused(call(y=None), -1, "y is NULL")
    refused(call(xo=None, h=None), -1, "both NULL")
    for key in ("x", "y", "xo", "h"):
        refused(call(**{key: 8}), -3, "not 16-byte")
    for h in (16, 32, 64):
        refused(call(h=h), -1, "overlaps")
    assert call(n=0, x=None, y=None) == 0
    refused(grad(xo=None), -1, "x_out")
    refused(grad(y=None), -1, "y is NULL")
    for key in ("xo", "dxo", "dh", "y", "dx", "dy"):
        refused(grad(**{key: 8}), -3, "not 16-byte")
    refused(grad(k=0), -1, "k = 0")
    refused(grad(dx=128), -1, "the same")
    need = lib.hmoe_join_workspace(join(), 10)
    assert need > 0
    refused(grad(wb=need - 1), -4, "workspace")
    refused(grad(ws=24), -3, "workspace")
    assert lib.hmoe_join_workspace(join(k=9), 10) == 0


def test_ortho_refusals(lib):
    big = 1 << 40
    good = (F * 3)(1.0, 2.0, 3.0)

    def ortho(G=16, dt=1, K=2, rows=16, cols=24, steps=5, coef=good, O=16, ws=16, wb=big):
        return lib.hmoe_orthogonalise(G, dt, K, rows, cols, steps, coef, O, ws, wb, None)

    def step(w=16, g=16, v=16, lo=32, dt=1, K=2, rows=16, cols=24, lr=0.1, wd=0.1, mu=0.9, scale=1.0, steps=5, coef=good, ws=16,
             wb=big):
        return lib.hmoe_muon_step(w, g, v, lo, dt, K, rows, cols, F(lr), F(wd), F(mu), 1, F(scale), steps, coef, ws, wb, None)

    for call in (ortho, step):
        refused(call(dt=3), -2, "dtype")
        refused(call(K=0), -1, "K =")
        refused(call(K=4097), -1, "K =")
        refused(call(rows=0), -1, "rows")
        refused(call(cols=20), -3, "cols")
        refused(call(cols=0), -3, "cols")
        refused(call(rows=(1 << 21) + 1), -1, "exceeds")
        refused(call(rows=1 << 16, cols=1 << 16), -1, "smaller")
        refused(call(steps=0), -1, "steps")
        refused(call(steps=33), -1, "steps")
        refused(call(coef=None), -1, "coef")
        for bad in (NAN, INF):
            refused(call(coef=(F * 3)(1.0, bad, 1.0)), -1, "coef")
        need = lib.hmoe_muon_workspace(2, 16, 24)
        assert need == lib.hmoe_orthogonalise_workspace(2, 16, 24, 1) > 0
        refused(call(wb=need - 1), -4, "workspace")
        refused(call(ws=None), -4, "workspace")
        refused(call(ws=24), -3, "workspace")
    for key in ("G", "O"):
        refused(ortho(**{key: None}), -1, key)
        refused(ortho(**{key: 24}), -3, key)
    for key in ("w", "g", "v"):
        refused(step(**{key: None}), -1, key)
        refused(step(**{key: 24}), -3, key)
    refused(step(lo=24), -3, "w_lo")
    refused(step(lo=16), -1, "w_lo")
    for key in ("lr", "wd", "mu"):
        for bad in (-0.1, NAN, INF):
            refused(step(**{key: bad}), -1, "negative")
    refused(step(scale=INF), -1, "scale")
    assert lib.hmoe_muon_workspace(0, 16, 24) == 0 and lib.hmoe_muon_workspace(1, 1 << 16, 1 << 16) == 0


def test_binding_refusals():
    X, R = torch.zeros(4, 16), torch.zeros(3, 16)
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.router_forward({"R": R}, X)
    with pytest.raises(hmoe.HmoeError, match="bias: shape"):
        hmoe.make_router({"R": R, "bias": torch.zeros(4)})
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.join_forward(X, X)
    with pytest.raises(hmoe.HmoeError, match="y: dtype"):
        hmoe.join_forward(X, X.bfloat16())
    with pytest.raises(hmoe.HmoeError, match="y: shape"):
        hmoe.join_forward(X, X[:3])
    with pytest.raises(hmoe.HmoeError, match="gate: shape"):
        hmoe.join_forward(X, X, gate=torch.zeros(4, 1))
    with pytest.raises(hmoe.HmoeError, match="gamma_h: dtype"):
        hmoe.join_forward(X, X, gamma_h=torch.zeros(16, dtype=torch.float64))
    with pytest.raises(hmoe.HmoeError, match="contiguous"):
        hmoe.join_forward(torch.zeros(16, 16).t(), X.repeat(4, 1))
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.join_backward(X, X, dx_out=X)
    with pytest.raises(hmoe.HmoeError, match="dx_out: shape"):
        hmoe.join_backward(X, X, dx_out=X[:2])
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.orthogonalise(X)
    with pytest.raises(hmoe.HmoeError, match="matrix"):
        hmoe.orthogonalise(X[0])
    with pytest.raises(hmoe.HmoeError, match="out: shape"):
        hmoe.orthogonalise(X, out=X[:2])
    with pytest.raises(hmoe.HmoeError, match="g: shape"):
        hmoe.muon_step(X, X[:2], X)
    with pytest.raises(hmoe.HmoeError, match="w: dtype"):
        hmoe.muon_step(X.bfloat16(), X, X)
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.muon_step(X, X, X)


def test_refuses_results_over_what_is_still_read(lib):
    big = 1 << 40
    good = (F * 3)(1.0, 2.0, 3.0)
    # dX is written before dR reads X
    rc = lib.hmoe_router_backward(ctypes.byref(router()), 10, 32, 16, 16, 16, 16, F(0.1), F(0.1), 32, 64, 16, 16, big, None)
    refused(rc, -1, "dX is X")
    # rows of y that another workgroup still reads
    rc = lib.hmoe_join_forward(join(k=2), 10, 16, 32, 16, 32, 64, None)
    refused(rc, -1, "x_out is y")

    def grad(k, dx, dy):
        return lib.hmoe_join_backward(join(k=k), 10, 256, 32, 16, 512, 1024, dx, dy, 16, 16, 16, 16, big, None)
    for k in (1, 2):
        refused(grad(k, 32, 128), -1, "dx is y")
    for dy in (256, 512, 1024):
        refused(grad(2, 64, dy), -1, "dy is")

    def step(w, g, v, lo, mu=0.9):
        return lib.hmoe_muon_step(w, g, v, lo, 1, 2, 16, 24, F(0.1), F(0.1), F(mu), 1, F(1.0), 5, good, 16, big, None)
    refused(step(16, 32, 32, None), -1, "v is")
    refused(step(16, 32, 16, None), -1, "v is")
    refused(step(16, 32, 64, 64), -1, "w_lo is")
    refused(step(16, 32, 64, 32), -1, "w_lo is")


def test_refuses_a_router_of_another_device():
    prm = router(K=3, d=16, top_k=1, dt=hmoe._DT[torch.float32])
    prm.device = 1
    with pytest.raises(hmoe.HmoeError, match="router on device 1"):
        hmoe._router(prm, torch.zeros(4, 16), 1, False)
