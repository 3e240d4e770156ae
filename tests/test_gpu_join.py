"""The join with the residual stream and its gradients against the formulas in 64 bits.

Bounds, element by element.  eps / 2 of a type is the largest relative error of one rounding.  A row's sums are made of
at most 32 additions in a lane and 10 across lanes and waves, so that one of terms t is off by at most 48 2^-24
sum |t|; a value made of sums and a dozen products and additions of fp32 by 96 2^-24 times the sum of the magnitudes
of its terms (`mag`), and what is stored in T by eps(T) / 2 of itself more.  Column sums over n rows are n / 1024
additions in a lane and 70 behind it at most: 256 2^-24 for the sizes here."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
EPS = 1e-5


def near(got, ref, mag, dtype, terms=96):
    half = torch.finfo(dtype).eps / 2
    off = np.abs(np64(got) - ref) - (half * np.abs(ref) + terms * U * mag * (1 + half) + 1e-30)
    assert off.max(initial=-1.0) <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))


def make(n, d, k, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[dtype])
    return {"x": r(n, d), "y": r(n, k, d), "gate": torch.randn(n, k, generator=g, device="cuda"), "gy": r(d) + 1,
            "gh": r(d) + 1, "dx_out": r(n, d), "dh": r(n, d)}


def forward64(x, y, gate, gy, gh, norm, scale):
    r = 1 / np.sqrt((y * y).mean(2, keepdims=True) + EPS) if norm else np.ones_like(y[:, :, :1])
    terms = gate[:, :, None] * (y * r * gy)
    new = scale * x + terms.sum(1)
    mag = np.abs(scale * x) + np.abs(terms).sum(1)
    rh = 1 / np.sqrt((new * new).mean(1, keepdims=True) + EPS)
    # an error of x' moves its norm by as much at most
    return new, mag, new * rh * gh, (mag + np.abs(new) * np.linalg.norm(mag, axis=1, keepdims=True)
                                     / np.maximum(np.linalg.norm(new, axis=1, keepdims=True), 1e-30)) * rh * np.abs(gh)


def backward64(xo, y, gate, gy, gh, norm, scale, dxo, dh):
    r = 1 / np.sqrt((xo * xo).mean(1, keepdims=True) + EPS)
    t = dh * gh
    D = dxo + r * (t - xo * r * r * (t * xo).mean(1, keepdims=True))
    mD = np.abs(dxo) + r * (np.abs(t) + np.abs(xo) * r * r * np.abs(t * xo).mean(1, keepdims=True))
    out = {"dx": (scale * D, np.abs(scale) * mD), "dgamma_h": ((dh * xo * r).sum(0), np.abs(dh * xo * r).sum(0))}
    D, mD = D[:, None, :], mD[:, None, :]
    ry = 1 / np.sqrt((y * y).mean(2, keepdims=True) + EPS) if norm else np.ones_like(y[:, :, :1])
    yn = y * ry
    s, ms = D * gy, mD * np.abs(gy)
    out["dgate"] = ((s * yn).sum(2), (ms * np.abs(yn)).sum(2))
    g3 = gate[:, :, None]
    out["dgamma_y"] = ((g3 * D * yn).sum((0, 1)), np.abs(g3 * mD * yn).sum((0, 1)))
    if norm:
        dy = g3 * ry * (s - yn * (s * yn).mean(2, keepdims=True))
        mdy = np.abs(g3) * ry * (ms + np.abs(yn) * (ms * np.abs(yn)).mean(2, keepdims=True))
    else:
        dy, mdy = g3 * s, np.abs(g3) * ms
    out["dy"] = (dy, mdy)
    return out


WIDTHS = [8, 24, 64, 72, 128, 200, 256, 264, 512, 520, 1000, 1024, 2048, 2056, 4104, 8192, 16392, 32768]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, dtype):
    n = 37 if d > 4096 else 301
    check(make(n, d, 1, dtype, d), True, 0.75, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,k,norm", [(1, 64, 1, True), (2, 2048, 8, True), (333, 96, 3, False), (5000, 64, 2, True),
                                        (2500, 1024, 2, False), (1, 8, 8, False), (3, 4096, 2, True)])
def test_rows_and_experts(n, d, k, norm, dtype):
    check(make(n, d, k, dtype, n + d), norm, -1.25, dtype)


def check(m, norm, scale, dtype):
    T = DT[dtype]
    q = {k: np64(v) for k, v in m.items()}
    how = dict(gate=m["gate"], gamma_y=m["gy"], gamma_h=m["gh"], norm_y=norm, scale=scale, eps=EPS)
    f = hmoe.join_forward(m["x"], m["y"], **how)
    new, mag, h, mag_h = forward64(q["x"], q["y"], q["gate"], q["gy"], q["gh"], norm, scale)
    near(f["x"], new, mag, T)
    near(f["h"], h, mag_h, T, 192)
    b = hmoe.join_backward(f["x"], m["y"], dx_out=m["dx_out"], dh=m["dh"], **how)
    ref = backward64(np64(f["x"]), q["y"], q["gate"], q["gy"], q["gh"], norm, scale, q["dx_out"], q["dh"])
    for key in ("dx", "dy"):
        near(b[key], *ref[key], T, 192)
    for key in ("dgate", "dgamma_y", "dgamma_h"):
        near(b[key], *ref[key], torch.float32, 512)


def test_what_is_not_given_or_wanted():
    m = make(50, 128, 2, "f32")
    q = {k: np64(v) for k, v in m.items()}
    one, none = np.ones(128), np.zeros((50, 128))
    f = hmoe.join_forward(m["x"], eps=EPS)  # the norm alone
    assert torch.equal(f["x"], m["x"])
    new, mag, h, mag_h = forward64(q["x"], np.zeros((50, 1, 128)), np.ones((50, 1)), one, one, True, 1.0)
    near(f["h"], h, mag_h, torch.float32)
    f = hmoe.join_forward(m["x"], m["y"], want_h=False, norm_y=False, eps=EPS)  # a plain sum
    assert f["h"] is None
    near(f["x"], q["x"] + q["y"].sum(1), np.abs(q["x"]) + np.abs(q["y"]).sum(1), torch.float32)
    f = hmoe.join_forward(m["x"], m["y"][:, 0].contiguous(), gate=m["gate"][:, 0].contiguous(), want_x=False, eps=EPS)
    assert f["x"] is None
    b = hmoe.join_backward(m["x"], m["y"], m["gate"], dx_out=m["dx_out"], eps=EPS)  # h was not used
    ref = backward64(q["x"], q["y"], q["gate"], one, one, True, 1.0, q["dx_out"], none)
    assert b["dgamma_h"] is None and b["dgamma_y"] is None
    assert torch.equal(b["dx"], m["dx_out"])
    near(b["dy"], *ref["dy"], torch.float32)
    near(b["dgate"], *ref["dgate"], torch.float32)
    b = hmoe.join_backward(m["x"], dh=m["dh"], gamma_h=m["gh"], eps=EPS)  # x' was not used but for h
    ref = backward64(q["x"], np.zeros((50, 1, 128)), np.ones((50, 1)), one, q["gh"], True, 1.0, none, q["dh"])
    near(b["dx"], *ref["dx"], torch.float32)
    near(b["dgamma_h"], *ref["dgamma_h"], torch.float32, 256)
    b = hmoe.join_backward(m["x"], m["y"], m["gate"], m["gy"], dx_out=m["dx_out"], want=("dgamma_y",), eps=EPS)
    ref = backward64(q["x"], q["y"], q["gate"], q["gy"], one, True, 1.0, q["dx_out"], none)
    assert all(v is None for k, v in b.items() if k != "dgamma_y")
    near(b["dgamma_y"], *ref["dgamma_y"], torch.float32, 256)
    b = hmoe.join_backward(m["x"], m["y"], m["gate"], m["gy"], eps=EPS)  # no gradient comes in
    for key in ("dx", "dy", "dgate", "dgamma_y"):
        assert not b[key].any()


def test_no_rows():
    m = make(0, 64, 1, "f32")
    f = hmoe.join_forward(m["x"], m["y"], m["gate"], m["gy"], m["gh"])
    assert f["x"].shape == (0, 64)
    out = {"dgamma_y": torch.full((64,), 7.0, device="cuda"), "dgamma_h": torch.full((64,), 7.0, device="cuda")}
    hmoe.join_backward(m["x"], m["y"], m["gate"], m["gy"], m["gh"], dx_out=m["dx_out"], dh=m["dh"], out=out)
    assert not out["dgamma_y"].any() and not out["dgamma_h"].any()


@pytest.mark.parametrize("d", [64, 1024, 4096])
def test_in_place(d):
    m = make(70, d, 1, "bf16")
    m["y"] = m["y"][:, 0].contiguous()
    m["gate"] = m["gate"][:, 0].contiguous()
    how = dict(gate=m["gate"], gamma_y=m["gy"], gamma_h=m["gh"], scale=0.5)
    f = hmoe.join_forward(m["x"], m["y"], **how)
    b = hmoe.join_backward(f["x"], m["y"], dx_out=m["dx_out"], dh=m["dh"], **how)
    x = m["x"].clone()
    g = hmoe.join_forward(x, m["y"], out={"x": x}, **how)
    assert torch.equal(g["x"], f["x"]) and torch.equal(g["h"], f["h"]) and g["x"].data_ptr() == x.data_ptr()
    for where in ("dx_out", "dh"):
        t = {"dx_out": m["dx_out"].clone(), "dh": m["dh"].clone()}
        y = m["y"].clone()
        c = hmoe.join_backward(f["x"], y, dx_out=t["dx_out"], dh=t["dh"], out={"dx": t[where], "dy": y}, **how)
        for key in b:
            assert torch.equal(b[key], c[key]), (where, key)


def test_rows_of_zeros_and_not_numbers_stay_in_their_rows():
    m = make(40, 256, 2, "bf16")
    m["x"][3] = 0
    m["y"][3] = 0
    clean = hmoe.join_forward(m["x"], m["y"], m["gate"], m["gy"], m["gh"])
    assert not clean["x"][3].any() and not clean["h"][3].any()
    m["y"][5, 1, 7] = float("nan")
    m["x"][6, 0] = float("inf")
    f = hmoe.join_forward(m["x"], m["y"], m["gate"], m["gy"], m["gh"])
    keep = [i for i in range(40) if i not in (5, 6)]
    for key in ("x", "h"):
        assert torch.equal(f[key][keep], clean[key][keep])
        assert torch.isnan(f[key][5].float()).all()
    assert f["x"][6, 0] == float("inf") and torch.isnan(f["h"][6, 0].float())
    b = hmoe.join_backward(f["x"], m["y"], m["gate"], m["gy"], m["gh"], dx_out=m["dx_out"], dh=m["dh"])
    for key in ("dx", "dy", "dgate"):
        assert torch.isfinite(b[key][keep].float()).all()


def test_against_differences():
    """The gradient of a fixed linear function of x' and h along random directions, from differences in 64 bits of the
    formula: their error is h^2 |f'''| and 2^-53 / h, below 1e-6; the fp32 gradient's below 1e-4 of the sum of its terms."""
    m = make(9, 64, 2, "f32", 5)
    q = {k: np64(v) for k, v in m.items()}
    how = dict(gate=m["gate"], gamma_y=m["gy"], gamma_h=m["gh"], norm_y=True, scale=0.7, eps=EPS)
    f = hmoe.join_forward(m["x"], m["y"], **how)
    b = hmoe.join_backward(f["x"], m["y"], dx_out=m["dx_out"], dh=m["dh"], **how)

    def value(p):
        new, _, h, _ = forward64(p["x"], p["y"], p["gate"], p["gy"], p["gh"], True, 0.7)
        return (new * q["dx_out"]).sum() + (h * q["dh"]).sum()

    rs = np.random.default_rng(0)
    for key, grad in (("x", "dx"), ("y", "dy"), ("gate", "dgate"), ("gy", "dgamma_y"), ("gh", "dgamma_h")):
        v = rs.standard_normal(q[key].shape)
        up, down = dict(q, **{key: q[key] + 1e-5 * v}), dict(q, **{key: q[key] - 1e-5 * v})
        want = (value(up) - value(down)) / 2e-5
        got = (np64(b[grad]) * v).sum()
        assert abs(got - want) <= 1e-4 * np.abs(np64(b[grad]) * v).sum(), (key, got, want)


def test_captured_and_replayed():
    m = make(100, 512, 2, "bf16")
    how = dict(gate=m["gate"], gamma_y=m["gy"], gamma_h=m["gh"])
    want_f = hmoe.join_forward(m["x"], m["y"], **how)
    want_b = hmoe.join_backward(want_f["x"], m["y"], dx_out=m["dx_out"], dh=m["dh"], **how)
    out_f = {k: torch.empty_like(v) for k, v in want_f.items()}
    out_b = {k: torch.empty_like(v) for k, v in want_b.items()}
    ws = torch.empty(hmoe.join_workspace(100, 512, 2, torch.bfloat16), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hmoe.join_forward(m["x"], m["y"], out=out_f, **how)
        hmoe.join_backward(out_f["x"], m["y"], dx_out=m["dx_out"], dh=m["dh"], out=out_b, ws=ws, **how)
    for _ in range(3):
        for t in (*out_f.values(), *out_b.values()):
            t.fill_(3)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in ((out_f, want_f), (out_b, want_b)):
            for k in want:
                assert torch.equal(got[k], want[k]), k
