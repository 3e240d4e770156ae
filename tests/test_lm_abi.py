"""The entry points of include/hmoe_lm.h: exported, bound, and refusing bad arguments before anything is
launched (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

from paper_1704_06363_amd import hmoe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hmoe.LIB_PATH):
        from paper_1704_06363_amd import build
        build.build()
    return hmoe.lib()


def refused(rc, code, word):
    assert rc == code and word in hmoe.last_error(), (rc, hmoe.last_error())


def test_exports_every_declared_symbol(lib):
    src = open(os.path.join(ROOT, "include", "hmoe_lm.h")).read()
    names = sorted(set(re.findall(r"\b(hmoe_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", src, flags=re.S))))
    assert set(names) == set(hmoe.LM_SYMBOLS)
    for name in names:
        assert hasattr(lib, name), name


def test_token_logprob_refusals(lib):
    def call(logits=16, ld=64, anchor=None, dt=1, n=10, vocab=64, scale=1.0, token=16, m=3, top=16, ws=None, wb=0):
        return lib.hmoe_token_logprob(logits, ld, anchor, dt, n, vocab, F(scale), token, m, 16, 16, 16, 16, top, 16, ws,
                                      wb, None)
    refused(call(logits=None), -1, "logits")
    refused(call(logits=17), -3, "aligned")
    refused(call(dt=9), -2, "dtype")
    refused(call(n=-1), -1, "n =")
    refused(call(vocab=0), -1, "vocab")
    refused(call(ld=63), -1, "ld")
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(call(scale=scale), -1, "scale")
    refused(call(m=17), -1, "m = 17")
    refused(call(m=-1), -1, "m = -1")
    refused(call(vocab=8, m=9), -1, "m = 9")
    refused(call(top=None), -1, "top_idx")
    refused(call(anchor=20), -3, "anchor")
    refused(call(anchor=16, ld=72), -3, "apart")
    refused(call(anchor=16, vocab=60, ld=60), -3, "vocab")
    refused(call(anchor=16, logits=18), -3, "aligned")
    refused(call(vocab=100000, ld=100000, n=1), -4, "workspace")
    assert call(n=0, logits=None) == 0
    assert lib.hmoe_token_logprob_workspace(1, 100000, 16, 1) > 0
    assert lib.hmoe_token_logprob_workspace(0, 100000, 16, 1) == 0

    def grad(logits=16, ld=64, anchor=None, token=16, stat=16, entropy=16, gl=16, ge=16, out=32, ldo=64):
        return lib.hmoe_token_logprob_backward(logits, ld, anchor, 1, 10, 64, F(1.0), token, stat, entropy, gl, ge, out,
                                               ldo, None)
    refused(grad(stat=None), -1, "stat")
    refused(grad(token=None), -1, "token")
    refused(grad(entropy=None), -1, "entropy")
    refused(grad(out=None), -1, "dlogits")
    refused(grad(out=33), -3, "aligned")
    refused(grad(ldo=63), -1, "ld_out")
    refused(grad(out=16, ldo=72), -1, "in place")
    refused(grad(out=16, anchor=16), -1, "in place")


def test_token_logprob_binding_refusals():
    x, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.token_logprob(x, t)
    with pytest.raises(hmoe.HmoeError, match="token: dtype"):
        hmoe.token_logprob(x, t.long())
    with pytest.raises(hmoe.HmoeError, match="token: shape"):
        hmoe.token_logprob(x, t[:3])
    with pytest.raises(hmoe.HmoeError, match="dtype"):
        hmoe.token_logprob(x.half(), t)
    with pytest.raises(hmoe.HmoeError, match="top_idx: shape"):
        hmoe.token_logprob(x, t, m=3, out={"top_idx": torch.zeros(4, 2, dtype=torch.int32)})
    with pytest.raises(hmoe.HmoeError, match="stat: shape"):
        hmoe.token_logprob_backward(x, t, torch.zeros(4), None, torch.zeros(4))


def test_moe_few_refusals(lib):
    def call(n=4, X=16, expert=16, weight=16, Y=16, ws=None, wb=0, **kw):
        a = dict(K=8, d_in=64, d_hid=128, d_out=64, top_k=2, dt=1, act=0, R=16, r_bias=16, W1=16, b1=None, W2=16,
                 b2=None)
        a.update(kw)
        p = hmoe.FewParams(*a.values())
        return lib.hmoe_moe_few(ctypes.byref(p), n, X, expert, weight, Y, ws, wb, None)
    assert lib.hmoe_moe_few(None, 1, 16, 16, 16, 16, None, 0, None) == -1
    refused(call(dt=5), -2, "dtype")
    refused(call(K=0), -1, "K = 0")
    refused(call(K=4097), -1, "K = 4097")
    refused(call(d_in=60), -3, "d_in")
    refused(call(d_hid=0), -3, "d_hid")
    refused(call(d_out=12), -3, "d_out")
    refused(call(top_k=0), -1, "top_k")
    refused(call(top_k=9, K=16), -1, "top_k")
    refused(call(top_k=3, K=2), -1, "top_k")
    refused(call(act=2), -1, "act")
    refused(call(n=65), -1, "n = 65")
    refused(call(n=-1), -1, "n = -1")
    refused(call(R=None), -1, "R")
    refused(call(W1=20), -3, "W1")
    refused(call(X=None), -1, "X")
    refused(call(expert=None), -1, "expert")
    refused(call(weight=None), -1, "weight")
    refused(call(Y=24), -3, "Y")
    refused(call(), -4, "workspace")
    assert call(n=0, X=None) == 0


def test_moe_few_binding_refusals():
    b = torch.bfloat16
    p = {"R": torch.zeros(3, 16, dtype=b), "r_bias": None, "W1": torch.zeros(3, 24, 16, dtype=b), "b1": None,
         "W2": torch.zeros(3, 8, 24, dtype=b), "b2": None}
    with pytest.raises(hmoe.HmoeError, match="activation"):
        hmoe.make_few_params(p, 1, "tanh")
    with pytest.raises(hmoe.HmoeError, match="W1: shape"):
        hmoe.make_few_params(p, 1, "silu")
    with pytest.raises(hmoe.HmoeError, match="r_bias: dtype"):
        hmoe.make_few_params(dict(p, r_bias=torch.zeros(3, dtype=b)))
    with pytest.raises(hmoe.HmoeError, match="R: shape"):
        hmoe.make_few_params(dict(p, R=torch.zeros(4, 16, dtype=b)))
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.make_few_params(p)


def test_lora_refusals(lib):
    ok = dict(E=8, d_in=64, d_out=128, rank=16, dt=1, W=16, b=None, A=16, B=16, scale=None)

    def prm(**kw):
        return hmoe.Lora(*dict(ok, **kw).values())

    def few(n=4, X=16, adapter=16, Y=16, **kw):
        return lib.hmoe_lora_few(ctypes.byref(prm(**kw)), n, X, adapter, Y, None, 0, None)

    def fwd(n=400, X=16, offsets=16, U=16, Y=16, **kw):
        return lib.hmoe_lora_forward(ctypes.byref(prm(**kw)), n, X, offsets, None, U, Y, None, 0, None)

    def bwd(n=400, X=16, offsets=16, U=16, dY=16, dX=16, dA=16, dB=16, **kw):
        return lib.hmoe_lora_backward(ctypes.byref(prm(**kw)), n, X, offsets, None, U, dY, dX, dA, dB, None, 0, None)
    for call in (few, fwd, bwd):
        refused(call(dt=3), -2, "dtype")
        refused(call(E=0), -1, "E = 0")
        refused(call(E=4097), -1, "E = 4097")
        refused(call(d_in=4), -3, "d_in")
        refused(call(d_out=0), -3, "d_out")
        refused(call(rank=12), -3, "rank")
        refused(call(rank=136), -1, "rank")
        refused(call(d_in=(1 << 21) + 8), -1, "exceeds")
        refused(call(n=-1), -1, "n =")
        refused(call(W=None), -1, "W")
        refused(call(A=24), -3, "A")
        refused(call(B=None), -1, "B")
        refused(call(X=None), -1, "X")
        refused(call(), -4, "workspace")
    assert lib.hmoe_lora_few(None, 1, 16, 16, 16, None, 0, None) == -1
    refused(few(n=65), -1, "n = 65")
    refused(few(adapter=None), -1, "adapter")
    refused(few(Y=8), -3, "Y")
    refused(fwd(n=(1 << 28) + 1), -1, "n =")
    refused(fwd(offsets=None), -1, "offsets")
    refused(fwd(U=None), -1, "U")
    refused(bwd(U=None), -1, "U")
    refused(bwd(dY=None), -1, "dY")
    refused(bwd(dX=8), -3, "dX")
    refused(bwd(dA=8), -3, "dA")
    assert few(n=0, X=None) == 0 and fwd(n=0, X=None) == 0
    assert lib.hmoe_lora_saved_width(24, 1) == 96 and lib.hmoe_lora_saved_width(24, 0) == 24


def test_lora_binding_refusals():
    b = torch.bfloat16
    p = {"W": torch.zeros(24, 16, dtype=b), "b": None, "A": torch.zeros(3, 8, 16, dtype=b),
         "B": torch.zeros(3, 24, 8, dtype=b), "scale": None}
    with pytest.raises(hmoe.HmoeError, match="B: shape"):
        hmoe.make_lora(dict(p, B=torch.zeros(3, 24, 16, dtype=b)))
    with pytest.raises(hmoe.HmoeError, match="A: dtype"):
        hmoe.make_lora(dict(p, A=torch.zeros(3, 8, 16)))
    with pytest.raises(hmoe.HmoeError, match="scale: dtype"):
        hmoe.make_lora(dict(p, scale=torch.zeros(3, dtype=b)))
    with pytest.raises(hmoe.HmoeError, match="GPU"):
        hmoe.make_lora(p)
