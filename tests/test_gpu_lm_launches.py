"""Problems of more workgroups than one launch holds (2^32 threads), in integers that every sum holds exactly."""
import pytest
import torch

from paper_1704_06363_amd import hmoe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h,o", [(1 << 19, 8), (8, 1 << 19)])
def test_more_experts_and_columns_than_a_launch_takes(h, o):
    """64 samples with eight experts of their own each: 512 groups of 32768 tiles of 16 outputs."""
    n, K, k, d = 64, 512, 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    code = torch.tensor([[1.0 if i >> b & 1 else -1.0 for b in range(6)] + [1.0, 1.0] for i in range(n)], device="cuda")
    X = code.bfloat16()
    ints = lambda *s: torch.randint(-1, 2, s, generator=g, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    p = {"R": X.repeat_interleave(k, 0).contiguous(), "r_bias": None, "W1": ints(K, h, d), "b1": None,
         "W2": ints(K, o, h), "b2": None}
    f = hmoe.moe_few(p, X, top_k=k)
    assert torch.equal(f["expert"].flatten().long(), torch.arange(K, device="cuda"))
    assert bool((f["weight"] == 0.125).all())
    for i in range(n):
        e = slice(k * i, k * i + k)
        hid = (p["W1"][e].float() * X[i].float()).sum(2).clamp_min_(0)
        y = torch.stack([(p["W2"][j].float() * hid[j - k * i]).sum(1, dtype=torch.float64) for j in range(k * i, k * i + k)])
        assert torch.equal(f["Y"][i], (y.sum(0) / k).float().bfloat16()), i


def test_as_many_rows_as_the_adapters_take():
    n, E, d, o, r = 1 << 28, 3, 8, 8, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    ints = lambda *s: torch.randint(-1, 2, s, generator=g, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    p = {"W": ints(o, d), "b": None, "A": ints(E, r, d), "B": ints(E, o, r), "scale": None}
    X = ints(n, d)
    off = torch.tensor([0, 100, n - 70000, n], dtype=torch.int32, device="cuda")
    Y = hmoe.lora_forward(p, X, off)["Y"]
    for first, last, e in ((0, 100, 0), (100, 5000, 1), (n - 75000, n - 70000, 1), (n - 70000, n, 2), (n - 64, n, 2)):
        x = X[first:last].float()
        ref = x @ p["W"].float().t() + x @ p["A"][e].float().t() @ p["B"][e].float().t()
        assert torch.equal(Y[first:last], ref.bfloat16()), (first, e)
