"""How the operators of hmoe_train.h may be called: what lies beside their outputs stays as it is, the same call gives the
same bits, on any stream, workspaces may be dirty and shared by the directions, and too small ones are refused."""
import pytest
import torch

from paper_1704_06363_amd import hmoe

pytestmark = pytest.mark.gpu

PAD = 64  # elements on either side of every buffer


class Guarded:
    """Tensors inside larger ones whose rest is checked."""

    def __init__(self):
        self.all = []

    def __call__(self, *shape, dtype=torch.float32):
        n = 1
        for s in shape:
            n *= s
        whole = torch.full((n + 2 * PAD,), 77, dtype=dtype, device="cuda")
        t = whole[PAD:PAD + n].view(*shape)
        t.zero_()
        self.all.append((whole, n))
        return t

    def check(self):
        torch.cuda.synchronize()
        for whole, n in self.all:
            assert (whole[:PAD] == 77).all() and (whole[PAD + n:] == 77).all(), (whole.dtype, n)


def dirty(nbytes):
    """A workspace of exactly nbytes inside a larger buffer, full of NaN bits."""
    whole = torch.full((nbytes + 512,), 255, dtype=torch.uint8, device="cuda")
    return whole, whole[256:256 + nbytes]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def router_call(n, K, d, top, dtype, seed):
    g = gen(seed)
    p = {"R": torch.randn(K, d, generator=g, device="cuda").to(dtype), "bias": torch.randn(K, generator=g, device="cuda")}
    X = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    gw = torch.randn(n, top, generator=g, device="cuda")
    i32 = torch.int32

    def call(b):
        whole, ws = dirty(hmoe.router_workspace(p, n, top))
        out = {"expert": b(n, top, dtype=i32), "weight": b(n, top), "scores": b(n, K), "counts": b(K, dtype=i32), "share": b(K),
               "loss": b(2)}
        f = hmoe.router_forward(p, X, top_k=top, out=out, ws=ws)
        r = hmoe.router_backward(p, X, f, gw, 0.1, 0.1, out={"dX": b(n, d, dtype=dtype), "dR": b(K, d), "dbias": b(K)}, ws=ws)
        return {**f, **r}, whole
    return call


def join_call(n, d, k, dtype, seed):
    g = gen(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)
    x, y, gy, gh, dxo, dh = r(n, d), r(n, k, d), r(d), r(d), r(n, d), r(n, d)
    gate = torch.rand(n, k, generator=g, device="cuda")
    how = dict(gate=gate, gamma_y=gy, gamma_h=gh)

    def call(b):
        whole, ws = dirty(hmoe.join_workspace(n, d, k, dtype))
        f = hmoe.join_forward(x, y, out={"x": b(n, d, dtype=dtype), "h": b(n, d, dtype=dtype)}, **how)
        out = {"dx": b(n, d, dtype=dtype), "dy": b(n, k, d, dtype=dtype), "dgate": b(n, k), "dgamma_y": b(d), "dgamma_h": b(d)}
        return {**f, **hmoe.join_backward(f["x"], y, dx_out=dxo, dh=dh, out=out, ws=ws, **how)}, whole
    return call


def muon_call(K, rows, cols, dtype, seed):
    g = gen(seed)
    r = lambda: torch.randn(K, rows, cols, generator=g, device="cuda")
    w0, g0, v0 = r(), r(), r()

    def call(b):
        whole, ws = dirty(hmoe.muon_workspace(K, rows, cols))
        w, v, lo = b(K, rows, cols), b(K, rows, cols), b(K, rows, cols, dtype=dtype)
        w.copy_(w0)
        v.copy_(v0)
        hmoe.muon_step(w, g0, v, w_lo=lo, ws=ws)
        o = b(K, rows, cols, dtype=dtype)
        G = g0.to(dtype)
        hmoe.orthogonalise(G, out=o, ws=ws)
        return {"w": w, "v": v, "lo": lo, "o": o}, whole
    return call


CALLS = [(router_call, (1, 3, 8, 1)), (router_call, (777, 8, 64, 1)), (router_call, (130, 33, 72, 5)),
         (router_call, (300, 130, 264, 8)), (router_call, (16501, 17, 24, 2)), (router_call, (515, 48, 520, 3)),
         (join_call, (1, 8, 1)), (join_call, (5, 72, 3)), (join_call, (333, 520, 2)), (join_call, (17, 4104, 1)),
         (join_call, (2049, 64, 8)), (join_call, (3, 32768, 2)),
         (muon_call, (1, 1, 8)), (muon_call, (3, 17, 24)), (muon_call, (2, 40, 1608)), (muon_call, (3, 777, 120)),
         (muon_call, (2, 129, 152)), (muon_call, (1, 1001, 200)), (muon_call, (23, 130, 264)), (muon_call, (1, 2500, 640)),
         (muon_call, (3, 513, 528))]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("make,size", CALLS)
def test_bounds_and_bits(make, size, dtype):
    call = make(*size, dtype, sum(size))
    b = Guarded()
    one, whole = call(b)
    b.check()
    assert (whole[:256] == 255).all() and (whole[-256:] == 255).all()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        two, _ = call(Guarded())
    stream.synchronize()
    for k in one:
        assert torch.equal(one[k], two[k]), k


def test_workspaces_that_are_too_small_are_refused():
    X, R = torch.zeros(100, 64, device="cuda"), torch.zeros(8, 64, device="cuda")
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.router_forward({"R": R}, X, ws=small)
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.join_backward(X, X, dx_out=X, ws=small)
    X = torch.zeros(200, 136, device="cuda")
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.orthogonalise(X, ws=small)
    with pytest.raises(hmoe.HmoeError, match="workspace"):
        hmoe.muon_step(X, X.clone(), X.clone(), ws=small)
    assert not X.any()


def test_two_calls_at_once_on_streams_of_their_own():
    calls = [router_call(2000, 40, 256, 2, torch.bfloat16, 1), muon_call(4, 300, 264, torch.bfloat16, 2),
             join_call(3000, 512, 2, torch.bfloat16, 3)]
    want = [c(Guarded())[0] for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for s, c in zip(streams, calls):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([c(Guarded())[0] for _ in range(3)])
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        for g in many:
            for k in w:
                assert torch.equal(w[k], g[k]), k
