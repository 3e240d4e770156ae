"""Measured cases of training a mixture whose router learns: the router with its balance losses, the
residual joins with their norms around a layer, and the orthogonalised update of weight matrices.

Each case is a dict of plain values; its "kind" names the operator:

  router  scores of every expert, the best of them with their weights, counts per expert and the
          balance and z losses; with "grad" the gradients of input, router rows and bias
  join    a residual connection: norm, gate and scale of what a layer gave, and the norm before the
          next layer; with "grad" the gradients of all that went in
  muon    a step of weight matrices: momentum, Newton-Schulz iterations towards the nearest
          orthogonal matrix, weight decay, and the weights in bf16
  ortho   the Newton-Schulz iterations alone, bf16 in and out

run() computes a case with elementary torch operations in 32 bits, or, where `own` is set, through
the public binding; exact() has the definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
COEF = (3.4445, -4.7750, 2.0315)  # of x, x^3 and x^5: a few steps take singular values of [0.01, 1] to about [0.7, 1.2]
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # The tiny configuration's features past a router of its eight experts, fp32, an odd number
        # of rows: launches are most of it.
        dict(name="router_tiny", kind="router", n=777, K=8, d=64, top=1, renorm=False, off=0.0, dtype="f32", grad=True),
        # A batch that is evaluated: two of the skewed configuration's 128 experts for each sample,
        # an eighth of the experts switched off.
        dict(name="router_eval", kind="router", n=4001, K=128, d=2048, top=2, renorm=True, off=0.125, dtype="bf16",
             grad=False),
        # The balanced configuration's training batch, one expert of 16 each.
        dict(name="router_balanced", kind="router", n=65536, K=16, d=2048, top=1, renorm=False, off=0.0, dtype="bf16",
             grad=True),
        # The skewed configuration's training batch, four of 128 experts each.
        dict(name="router_skewed", kind="router", n=32768, K=128, d=2048, top=4, renorm=True, off=0.0, dtype="bf16",
             grad=True),
        # One sample that is being answered, between two layers of the balanced configuration's width.
        dict(name="join_one", kind="join", n=1, d=2048, k=1, gated=True, norm=True, after=True, scale=1.0,
             dtype="bf16", grad=False),
        # The tiny configuration's width in fp32, odd rows, forward and backward.
        dict(name="join_tiny", kind="join", n=777, d=64, k=1, gated=True, norm=True, after=True, scale=0.5,
             dtype="f32", grad=True),
        # The balanced configuration's training batch between two layers.
        dict(name="join_balanced", kind="join", n=65536, d=2048, k=1, gated=True, norm=True, after=True, scale=1.0,
             dtype="bf16", grad=True),
        # Two experts' answers for each sample of the skewed configuration, joined by their weights.
        dict(name="join_pairs", kind="join", n=16384, d=1024, k=2, gated=True, norm=False, after=True, scale=1.0,
             dtype="bf16", grad=True),
        # First layers of the tiny configuration's eight experts: launches are all of it.
        dict(name="muon_tiny", kind="muon", K=8, rows=128, cols=64, nesterov=True, decay=0.01),
        # Three matrices of odd proportions.
        dict(name="muon_odd", kind="muon", K=3, rows=1001, cols=200, nesterov=False, decay=0.0),
        # The decoder of the balanced configuration, one very tall matrix.
        dict(name="muon_decoder", kind="muon", K=1, rows=50000, cols=1024, nesterov=True, decay=0.01),
        # First layers of the balanced configuration's 16 experts, gradients and updates in bf16.
        dict(name="ortho_experts", kind="ortho", K=16, rows=4096, cols=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    return max(8, _log(rng, lo, hi) // 8 * 8)


def _draw_router(rng):
    K = _log(rng, 3, 512)
    return dict(kind="router", n=_log(rng, 16, 65536), K=K, d=_width(rng, 64, 2048),
                top=min(K - 1, rng.choice([1, 1, 2, 3, 4, 8])), renorm=rng.random() < 0.5,
                off=rng.choice([0.0, 0.0, 0.2]) if K >= 16 else 0.0, dtype=rng.choice(["bf16", "bf16", "f32"]),
                grad=rng.random() < 0.7)


def _draw_join(rng):
    return dict(kind="join", n=_log(rng, 1, 65536), d=_width(rng, 64, 8192), k=rng.choice([1, 1, 1, 2, 4]),
                gated=rng.random() < 0.6, norm=rng.random() < 0.6, after=rng.random() < 0.8,
                scale=rng.choice([1.0, 1.0, rng.uniform(0.3, 1.5)]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                grad=rng.random() < 0.6)


def _draw_muon(rng):
    return dict(kind="muon", K=_log(rng, 1, 32), rows=_log(rng, 16, 4096), cols=_width(rng, 16, 4096),
                nesterov=rng.random() < 0.6, decay=rng.choice([0.0, 0.01]))


def _draw_ortho(rng):
    return dict(kind="ortho", K=_log(rng, 1, 32), rows=_log(rng, 16, 4096), cols=_width(rng, 16, 4096))


def draw(rng):
    kind = rng.choice(["router", "join", "muon", "ortho"])
    most = [work(c) for c in listed() if c["kind"] == kind]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        c = {"router": _draw_router, "join": _draw_join, "muon": _draw_muon, "ortho": _draw_ortho}[kind](rng)
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def work(case):
    c = case
    if c["kind"] == "router":
        b, n, K, d, top = BYTES[c["dtype"]], c["n"], c["K"], c["d"], c["top"]
        forward = b * (n * d + K * d) + 4 * K + 4 * n * K + 8 * n * top + 8 * K + 8
        if not c["grad"]:
            return {"bytes": forward, "flops": 2 * n * K * d}
        # the input is read once for both directions; its gradient, the rows' and the bias's are written
        return {"bytes": forward + b * n * d + 4 * n * top + 4 * K * d + 4 * K, "flops": 6 * n * K * d}
    if c["kind"] == "join":
        b, n, d, k = BYTES[c["dtype"]], c["n"], c["d"], c["k"]
        gate = 4 * n * k if c["gated"] else 0
        gains = b * d * (int(c["norm"]) + int(c["after"]))
        forward = b * n * d * (1 + k + 1 + int(c["after"])) + gate + gains
        if not c["grad"]:
            return {"bytes": forward, "flops": 10 * n * d * (k + 1)}
        # in: two gradients; out: those of x and y
        backward = b * n * d * (1 + int(c["after"]) + 1 + k) + gate + 4 * d * (int(c["norm"]) + int(c["after"]))
        return {"bytes": forward + backward, "flops": 30 * n * d * (k + 1)}
    K, r, l = c["K"], min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    # a step: X X^T and its square, which are symmetric, and a product with X
    flops = 5 * K * (r * r * l + r * r * r + 2 * r * r * l)
    size = K * r * l
    return {"bytes": size * (4 * 3 + 4 * 2 + 2 if c["kind"] == "muon" else 4), "flops": flops}


# ------------------------------------------------------------------ inputs

def _randn(shape, g, dtype, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


def _prepare_router(c, g):
    n, K, d, top, dt = c["n"], c["K"], c["d"], c["top"], DT[c["dtype"]]
    # a learned router's rows and small biases; experts that are off have a bias of -inf
    R = _randn((K, d), g, dt, 2.0 * d ** -0.5)
    bias = torch.randn(K, generator=g, device=DEV) * 0.05
    off = torch.randperm(K, generator=g, device=DEV)[:min(int(K * c["off"]), K - top - 1)]
    bias[off] = float("-inf")
    X = _randn((n + n // 2 + 8, d), g, dt)
    # A sample whose choice hangs on the last bits of its scores has no answer to compare: such are
    # passed over, of more samples than wanted.
    s = (X.double() @ R.double().t() + bias.double()).topk(top + 1, 1)[0]
    near = (s[:, :-1] - s[:, 1:] < 1e-5 * s.abs().amax()).any(1)
    X = X[torch.sort(near.int(), stable=True)[1][:n]].contiguous()
    st = {"case": c, "p": {"R": R, "bias": bias}, "X": X}
    if c["grad"]:
        st["g_weight"] = torch.randn(n, top, generator=g, device=DEV) / n
    if own:
        from paper_1704_06363_amd import hmoe
        f = lambda *s: torch.empty(*s, device=DEV)
        i = lambda *s: torch.empty(*s, device=DEV, dtype=torch.int32)
        st["ws"] = torch.empty(max(hmoe.router_workspace(st["p"], n, top), 1), dtype=torch.uint8, device=DEV)
        st["out"] = {"expert": i(n, top), "weight": f(n, top), "scores": f(n, K), "counts": i(K), "share": f(K),
                     "loss": f(2)}
        if c["grad"]:
            st["gout"] = {"dX": torch.empty(n, d, device=DEV, dtype=dt), "dR": f(K, d), "dbias": f(K)}
    return st


def _prepare_join(c, g):
    n, d, k, dt = c["n"], c["d"], c["k"], DT[c["dtype"]]
    st = {"case": c, "x": _randn((n, d), g, dt), "y": _randn((n, k, d), g, dt, 0.7), "gate": None, "gamma_y": None,
          "gamma_h": None, "dx_out": None, "dh": None}
    if c["gated"]:
        st["gate"] = torch.rand(n, k, generator=g, device=DEV)
    if c["norm"]:
        st["gamma_y"] = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(dt)
    if c["after"]:
        st["gamma_h"] = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(dt)
    if c["grad"]:
        st["dx_out"] = _randn((n, d), g, dt)
        if c["after"]:
            st["dh"] = _randn((n, d), g, dt)
        # the rows that an earlier forward kept for the backward: the sums that a pass makes anew could round the
        # other way in their last bit
        st["kept"] = _joined(st).to(dt)
    if own:
        from paper_1704_06363_amd import hmoe
        f = lambda *s: torch.empty(*s, device=DEV)
        e = lambda *s: torch.empty(*s, device=DEV, dtype=dt)
        st["out"] = {"x": e(n, d), "h": e(n, d) if c["after"] else None}
        if c["grad"]:
            st["gout"] = {"dx": e(n, d), "dy": e(n, k, d), "dgate": f(n, k) if c["gated"] else None,
                          "dgamma_y": f(d) if c["norm"] else None, "dgamma_h": f(d) if c["after"] else None}
            st["ws"] = torch.empty(max(hmoe.join_workspace(n, d, k, dt), 1), dtype=torch.uint8, device=DEV)
    return st


def _gradients(K, rows, cols, g):
    """Gradients as they are met: a few directions that many samples share, and a floor of noise; sizes that
    differ from matrix to matrix."""
    out = torch.empty(K, rows, cols, device=DEV)
    q = max(1, min(rows, cols) // 8)
    for m in out:
        a = torch.randn(rows, q, generator=g, device=DEV) * torch.linspace(1.0, 0.1, q, device=DEV)
        m.copy_(torch.randn(rows, cols, generator=g, device=DEV)).mul_(0.3)
        m.add_(a @ torch.randn(q, cols, generator=g, device=DEV), alpha=q ** -0.5)
    return out.mul_(1e-3 * torch.exp(torch.randn(K, 1, 1, generator=g, device=DEV)))


def _prepare_muon(c, g):
    K, rows, cols = c["K"], c["rows"], c["cols"]
    st = {"case": c, "g": _gradients(K, rows, cols, g)}
    st["v"] = torch.randn(K, rows, cols, generator=g, device=DEV).mul_(st["g"].std() * 2.0).add_(st["g"], alpha=4.0)
    st["w"] = torch.randn(K, rows, cols, generator=g, device=DEV).mul_(cols ** -0.5)
    st["w_lo"] = st["w"].to(torch.bfloat16)
    st["lr"], st["mu"], st["scale"] = 0.02, 0.95, max(1.0, rows / cols) ** 0.5
    if own:
        from paper_1704_06363_amd import hmoe
        st["ws"] = torch.empty(max(hmoe.muon_workspace(K, rows, cols), 1), dtype=torch.uint8, device=DEV)
    return st


def _prepare_ortho(c, g):
    K, rows, cols = c["K"], c["rows"], c["cols"]
    st = {"case": c, "G": _gradients(K, rows, cols, g).to(torch.bfloat16)}
    if own:
        from paper_1704_06363_amd import hmoe
        st["out"] = torch.empty_like(st["G"])
        st["ws"] = torch.empty(max(hmoe.orthogonalise_workspace(K, rows, cols, torch.bfloat16), 1), dtype=torch.uint8,
                               device=DEV)
    return st


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return {"router": _prepare_router, "join": _prepare_join, "muon": _prepare_muon,
            "ortho": _prepare_ortho}[case["kind"]](case, g)


BALANCE, Z = 0.01, 0.001  # weights of the router's two losses


# ------------------------------------------------------------------ one pass

def _key(x):
    """int64 keys [.., K] in the order (value descending, index ascending) of fp32 values, largest first."""
    K = x.shape[-1]
    i = (x + 0.0).view(torch.int32)
    i = torch.where(i < 0, i ^ 0x7FFFFFFF, i).long()
    return (i << 32) + (K - 1 - torch.arange(K, device=x.device))


def _plain_router(st):
    c, X, R = st["case"], st["X"].float(), st["p"]["R"].float()
    n, K, top = c["n"], c["K"], c["top"]
    s = X @ R.t() + st["p"]["bias"]
    idx = K - 1 - (torch.topk(_key(s), top, dim=1)[0] & 0xFFFFFFFF)
    mx = s.amax(1, keepdim=True)
    e = (s - mx).exp()
    tot = e.sum(1, keepdim=True)
    p = e / tot
    lse = (mx + tot.log())[:, 0]
    w = p.gather(1, idx)
    if c["renorm"]:
        best = (s.gather(1, idx) - mx).exp()
        w = best / best.sum(1, keepdim=True)
    hot = torch.zeros(n, K, device=DEV).scatter_(1, idx, 1.0)
    counts = hot.sum(0)
    share = p.double().sum(0).div(n).float()
    balance = K * (counts / (n * top) * share).sum()
    out = {"expert": idx.to(torch.int32), "weight": w, "scores": s, "counts": counts.to(torch.int32), "share": share,
           "loss": torch.stack([balance, lse.double().square().mean().float()])}
    if c["grad"]:
        gw = st["g_weight"]
        dp = (BALANCE * K / n) * (counts / (n * top)).expand(n, K).contiguous()
        if not c["renorm"]:
            dp.scatter_add_(1, idx, gw)
        ds = p * (dp - (p * dp).sum(1, keepdim=True)) + (2.0 * Z / n) * lse[:, None] * p
        if c["renorm"]:
            ds.scatter_add_(1, idx, w * (gw - (w * gw).sum(1, keepdim=True)))
        out.update(dX=(ds @ R).to(st["X"].dtype), dR=ds.t() @ X, dbias=ds.double().sum(0).float())
    return out


def _parts(st):
    """The rows of y in 32 bits, their norms' factors, gains and gates."""
    c, y = st["case"], st["y"].float()
    ry = (y.square().mean(2, keepdim=True) + EPS).rsqrt() if c["norm"] else 1.0
    return y, ry, st["gamma_y"].float() if c["norm"] else 1.0, st["gate"][:, :, None] if c["gated"] else 1.0


def _joined(st):
    y, ry, gy, gate = _parts(st)
    return st["case"]["scale"] * st["x"].float() + (gate * (y * ry * gy)).sum(1)


def _plain_join(st):
    c, dt = st["case"], st["x"].dtype
    x = _joined(st)
    out = {"x": x.to(dt), "h": None}
    if c["after"]:
        gh = st["gamma_h"].float()
        out["h"] = (x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * gh).to(dt)
    if c["grad"]:
        y, ry, gy, gate = _parts(st)
        yn = y * ry
        D = st["dx_out"].float()
        if c["after"]:
            xs = st["kept"].float()
            r = (xs.square().mean(1, keepdim=True) + EPS).rsqrt()
            xn = xs * r
            dh = st["dh"].float()
            out["dgamma_h"] = (dh * xn).double().sum(0).float()
            t = dh * gh
            D = D + r * (t - xn * (t * xn).mean(1, keepdim=True))
        out["dx"] = (c["scale"] * D).to(dt)
        D = D[:, None, :]
        if c["gated"]:
            out["dgate"] = (D * (yn * gy)).sum(2)
        t = D * gate * gy
        if c["norm"]:
            out["dgamma_y"] = (D * gate * yn).double().sum((0, 1)).float()
            t = ry * (t - yn * (t * yn).mean(2, keepdim=True))
        out["dy"] = t.expand(y.shape).to(dt)
    return out


def _newton_schulz(u):
    """fp32 [K, rows, cols] with rows <= cols."""
    X = u / u.double().square().sum((1, 2), keepdim=True).sqrt().float()
    for _ in range(5):
        A = X @ X.transpose(1, 2)
        X = COEF[0] * X + (COEF[1] * A + COEF[2] * (A @ A)) @ X
    return X


def _orthogonal(u):
    if u.shape[1] > u.shape[2]:
        return _newton_schulz(u.transpose(1, 2).contiguous()).transpose(1, 2)
    return _newton_schulz(u)


def _plain_muon(st):
    c, w, v, g = st["case"], st["w"], st["v"], st["g"]
    v.mul_(st["mu"]).add_(g)
    O = _orthogonal(g + st["mu"] * v if c["nesterov"] else v)
    w.mul_(1.0 - st["lr"] * c["decay"]).sub_(O, alpha=st["lr"] * st["scale"])
    st["w_lo"].copy_(w)
    return {"w": w, "v": v, "w_lo": st["w_lo"]}


def _own_router(st):
    from paper_1704_06363_amd import hmoe
    c, p = st["case"], st["p"]
    out = hmoe.router_forward(p, st["X"], top_k=c["top"], renorm=c["renorm"], out=st["out"], ws=st["ws"])
    if c["grad"]:
        out = dict(out, **hmoe.router_backward(p, st["X"], out, g_weight=st["g_weight"], balance=BALANCE, z=Z,
                                               renorm=c["renorm"], out=st["gout"], ws=st["ws"]))
    return out


def _own_join(st):
    from paper_1704_06363_amd import hmoe
    c = st["case"]
    how = dict(gate=st["gate"], gamma_y=st["gamma_y"], gamma_h=st["gamma_h"], norm_y=c["norm"], scale=c["scale"], eps=EPS)
    out = hmoe.join_forward(st["x"], st["y"], want_h=c["after"], out=st["out"], **how)
    if c["grad"]:
        out = dict(out, **hmoe.join_backward(st["kept"], st["y"], dx_out=st["dx_out"], dh=st["dh"], out=st["gout"],
                                             ws=st["ws"], **how))
    return out


def _own_muon(st):
    from paper_1704_06363_amd import hmoe
    c = st["case"]
    hmoe.muon_step(st["w"], st["g"], st["v"], lr=st["lr"], weight_decay=c["decay"], momentum=st["mu"],
                   nesterov=c["nesterov"], scale=st["scale"], coef=COEF, steps=5, w_lo=st["w_lo"], ws=st["ws"])
    return {"w": st["w"], "v": st["v"], "w_lo": st["w_lo"]}


def _own_ortho(st):
    from paper_1704_06363_amd import hmoe
    return {"O": hmoe.orthogonalise(st["G"], steps=5, coef=COEF, out=st["out"], ws=st["ws"])}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"router": _own_router, "join": _own_join, "muon": _own_muon, "ortho": _own_ortho}[kind](state)
    if kind == "ortho":
        return {"O": _orthogonal(state["G"].float()).to(torch.bfloat16)}
    return {"router": _plain_router, "join": _plain_join, "muon": _plain_muon}[kind](state)


# ------------------------------------------------------------------ 64 bits

def _exact_router(c, st):
    n, K, top = c["n"], c["K"], c["top"]
    X, R, b = (t.double().requires_grad_(c["grad"]) for t in (st["X"], st["p"]["R"], st["p"]["bias"]))
    s = torch.nn.functional.linear(X, R) + b
    idx = torch.argsort(s.detach(), dim=1, descending=True, stable=True)[:, :top]
    logp = torch.log_softmax(s, 1)
    w = torch.softmax(s.gather(1, idx), 1) if c["renorm"] else logp.gather(1, idx).exp()
    share = logp.exp().mean(0)
    counts = torch.bincount(idx.flatten(), minlength=K)
    balance = K * torch.dot(counts.double() / (n * top), share)
    z = torch.logsumexp(s, 1).pow(2).mean()
    out = {"expert": idx.to(torch.int32), "weight": w, "scores": s, "counts": counts.to(torch.int32), "share": share,
           "loss": torch.stack([balance, z])}
    if c["grad"]:
        total = (w * st["g_weight"].double()).sum() + BALANCE * balance + Z * z
        out["dX"], out["dR"], db = torch.autograd.grad(total, (X, R, b))
        out["dbias"] = torch.where(b.detach() == float("-inf"), 0.0, db)
    return out


def _exact_join(c, st):
    def unit(t):
        return t / torch.sqrt((t * t).sum(-1, keepdim=True) / t.shape[-1] + EPS)

    d = lambda k: st[k].double().requires_grad_() if st[k] is not None else None
    x, y, gate, gy, gh = d("x"), d("y"), d("gate"), d("gamma_y"), d("gamma_h")
    z = unit(y) if c["norm"] else y
    if gy is not None:
        z = z * gy
    if gate is not None:
        z = torch.einsum("nkd,nk->nkd", z, gate)
    new = c["scale"] * x + z.sum(1)
    out = {"x": new.detach(), "h": (unit(new) * gh).detach() if c["after"] else None}
    if c["grad"]:
        up = st["dx_out"].double()
        if c["after"]:  # through the norm of the kept row
            kept = d("kept")
            gk, out["dgamma_h"] = torch.autograd.grad(unit(kept) * gh, (kept, gh), st["dh"].double())
            up = up + gk
        names = [(k, t) for k, t in (("dx", x), ("dy", y), ("dgate", gate), ("dgamma_y", gy)) if t is not None]
        out.update(zip([k for k, _ in names], torch.autograd.grad(new, [t for _, t in names], up)))
    return out


def _exact_iterations(u):
    tall = u.shape[0] > u.shape[1]
    X = u / torch.linalg.matrix_norm(u)
    for _ in range(5):
        if tall:  # the polynomial of X^T X on the right
            S = X.mT @ X
            X = COEF[0] * X + X @ (COEF[1] * S + COEF[2] * (S @ S))
        else:
            S = X @ X.mT
            X = COEF[0] * X + (COEF[1] * S + COEF[2] * (S @ S)) @ X
    return X


def _exact_muon(c, st):
    v = st["mu"] * st["v"].double() + st["g"].double()
    u = st["g"].double() + st["mu"] * v if c["nesterov"] else v
    O = torch.stack([_exact_iterations(m) for m in u])
    w = (1.0 - st["lr"] * c["decay"]) * st["w"].double() - st["lr"] * st["scale"] * O
    return {"w": w, "v": v, "w_lo": w}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "ortho":
        return {"O": torch.stack([_exact_iterations(m.double()) for m in st["G"]])}
    return {"router": _exact_router, "join": _exact_join, "muon": _exact_muon}[case["kind"]](case, st)
