"""Token log-probabilities of rows that the usual ones do not show: blocks of NaN, anchored logits of a large
size, tokens that are masked, the largest scale.

Tolerances as in test_gpu_logprob.py, whose plain forms these tests use."""
import numpy as np
import pytest
import torch

from paper_1704_06363_amd import hmoe
from tests.parity import np64
from tests.test_gpu_logprob import DT, INF, check, check_grad, rows, tokens

pytestmark = pytest.mark.gpu


def blocks_of_nan(n, V, dtype, seed):
    """Rows with NaN in their first half, their first 2048 columns, alternate blocks of 1024, the first two
    entries of each eight, and all but the last five."""
    x = rows(n, V, 0, dtype, seed).clone()
    v = torch.arange(V, device="cuda")
    for i in range(0, n, 5):
        x[i, : V // 2] = float("nan")
        x[i + 1, : min(2048, V - 9)] = float("nan")
        x[i + 2, v // 1024 % 2 == 0] = float("nan")
        x[i + 3, v % 8 < 2] = float("nan")
        x[i + 4, : V - 5] = float("nan")
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(5, 700), (5, 8192), (5, 50000), (600, 20000), (1100, 5003)])
@pytest.mark.parametrize("m", [1, 9, 16])
def test_blocks_of_nan_rank_last(dtype, n, V, m):
    """A row in several pieces, in one of four waves, in one of one wave."""
    check(blocks_of_nan(n, V, dtype, V + m), tokens(n, V, m), m, 1.0)


@pytest.mark.parametrize("dtype,n,V,size", [("bf16", 12, 1000, 1e3), ("f32", 12, 1000, 1e4), ("bf16", 6, 30000, 1e4),
                                            ("f32", 600, 24000, 3e3), ("bf16", 1100, 520, 1e4)])
def test_anchored_logits_of_any_size(dtype, n, V, size):
    """A logit is anchor + stored value rounded to fp32, at 10^4 to 5e-4: the sums and the gradient take that number."""
    rs = np.random.default_rng(V)
    nb, tiles = -(-V // hmoe.ANCHOR_COLS), hmoe.anchor_shape(n, V)[0]
    a = np.full((n, tiles * 4), -3.0e38, np.float32)
    a[:, :nb] = size * rs.choice([1.0, 1.0003, 0.9998], (n, 1)) + rs.standard_normal((n, nb))
    anchor = torch.tensor(a.reshape(n, tiles, 4).transpose(1, 0, 2).copy()).cuda()
    x = torch.tensor(-np.abs(rs.standard_normal((n, V)) * 3)).to(DT[dtype]).cuda()
    full = (np.repeat(a[:, :nb], hmoe.ANCHOR_COLS, 1)[:, :V] + np64(x).astype(np.float32)).astype(np.float64)
    t = tokens(n, V, 1)
    f, lp, ent = check(x, t, 6, 1.0, anchor=anchor, full=full)
    check_grad(x, t, 1.0, f, lp, ent, 2, anchor=anchor)


@pytest.mark.parametrize("dtype,n,V", [("bf16", 6, 100), ("f32", 3, 9000)])
def test_a_masked_token(dtype, n, V):
    """Its log-probability is -inf, and its own entry of the gradient scale * g_logp as the formula has it: the one
    masked entry that is not 0."""
    x, t = rows(n, V, 0, dtype, 1).clone(), tokens(n, V, 2)
    at = t.long()[:, None]
    x.scatter_(1, at, -INF)
    x[:, V // 2::3] = -INF
    x[:, 0] = 1.0
    t[t == 0] = V // 2
    f, lp, ent = check(x, t, 4, 1.5)
    assert (np64(f["logp"]) == -INF).all()
    check_grad(x, t, 1.5, f, lp, ent, 3)
    g = torch.randn(n, device="cuda")
    d = hmoe.token_logprob_backward(x, t, f["stat"], f["entropy"], g, g, scale=1.5)
    own = d.gather(1, t.long()[:, None])[:, 0]
    assert torch.equal(own, (1.5 * g).to(x.dtype))
    masked = (x == -INF).scatter_(1, t.long()[:, None], False)
    assert bool((d[masked] == 0).all())


@pytest.mark.parametrize("dtype,n,V", [("bf16", 5, 700), ("f32", 3, 30000)])
def test_the_largest_scale(dtype, n, V):
    """Multiples of 2^-6: every entry but the largest has probability 0."""
    x, t = rows(n, V, 0, dtype, 1, ties=True) / 64, tokens(n, V, 2)
    check(x, t, 5, 2.0 ** 127)


@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_gradients_of_tokens_that_are_nearly_certain(scale):
    """Rows of two entries, p of the first 1 - e with e from 1e-2 to 1e-5: its gradient is 1 - p, and p carries
    the rounding of S = 1 + e (2^-24), v_exp_f32's last place (2^-23) and that of its argument and of the difference
    (2^-24 each, at most): 2.5 2^-23 of the gradient of logp."""
    n = 4000
    x = torch.zeros(n, 2, device="cuda")
    x[:, 1] = -torch.linspace(4.6, 11.5, n, device="cuda") / scale
    t = torch.zeros(n, dtype=torch.int32, device="cuda")
    f = hmoe.token_logprob(x, t, scale=scale)
    g = np64(hmoe.token_logprob_backward(x, t, f["stat"], None, torch.ones(n, device="cuda"), scale=scale))
    e = np.exp(scale * np64(x)[:, 1])
    ref = scale * (e / (1 + e))
    assert np.abs(g[:, 0] - ref).max() <= scale * 2.5 * 2.0 ** -23
