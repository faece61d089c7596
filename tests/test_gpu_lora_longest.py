"""dcut_lora at the largest K that it takes: where a row's bytes no longer fit 31 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_first_the_last_and_some_elements_of_the_longest_rows():
    """One adapter of rank 8 (17 GB); whole numbers, so that the result is exact."""
    from paper_2607_14647_b200 import binding
    K, N, bf16 = 1 << 30, 16, torch.bfloat16
    x, a = torch.zeros((1, K), dtype=bf16, device="cuda"), torch.zeros((1, 8, K), dtype=bf16, device="cuda")
    places = [0, 1, 7, 8, 63, 64, K // 8, K // 2 - 1, K // 2, K - 8, K - 1]
    for i, p in enumerate(places):
        x[0, p] = 1.0
        a[0, i % 8, p] = 2.0 ** (i // 8)
    s = torch.zeros(8)
    for i in range(len(places)):
        s[i % 8] += 2.0 ** (i // 8)
    b = (torch.arange(N * 8) % 5).float().view(1, N, 8)
    cu, zero = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 1], [0]))
    ctx = binding.Context(max_B=1, max_gamma=1)
    out = ctx.lora(x, a, b.to(bf16).cuda(), zero, torch.zeros((1, N), dtype=bf16, device="cuda"), cu, 1)
    assert ctx.poll_device_status() == 0
    assert torch.equal(out[0].float().cpu(), b[0] @ s)
