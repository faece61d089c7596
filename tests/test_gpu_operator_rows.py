"""What a row of the 8-bit and adapter operators depends on: itself and its own scales and adapter, bit for bit."""
import numpy as np
import pytest
import torch

from tests import test_gpu_linear8 as lin8
from tests import test_gpu_lora as adapters

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,N,K", [(130, 96, 200), (9, 500, 4096), (700, 300, 2176)])
@pytest.mark.parametrize("gated", [False, True])
def test_infinite_scales_stay_in_their_row_and_column(T, N, K, gated):
    """Infinite scales of one row, one column and, gated, one column of the second weight: every other element keeps its bits, those are no
    finite numbers (a sum that is 0, or a gate that is, gives NaN)."""
    ctx, c = lin8.context(), lin8.make(T + N, T, T, N, K, gated, bias=True)
    want = lin8.run(ctx, c).clone()
    row, cols = T - 3, [5] + ([N - 1] if gated else [])
    c["a_scale"][row] = float("inf")
    c["w_scale"][cols[0]] = float("inf")
    if gated:
        c["w2_scale"][cols[1]] = float("inf")
    got = lin8.run(ctx, c)
    keep_r, keep_c = [r for r in range(T) if r != row], [n for n in range(N) if n not in cols]
    assert torch.equal(got[keep_r][:, keep_c], want[keep_r][:, keep_c])
    assert not torch.isfinite(got[row].float()).any() and not torch.isfinite(got[:, cols].float()).any()


@pytest.mark.parametrize("counts,rank,gated", [([9, 17, 5, 1], 16, False), ([9, 17, 5, 1], 40, True), ([100, 64, 90, 30], 64, True), ([120, 3, 300, 65], 24, False),
                                               ([700, 100, 80, 9], 96, False)])
def test_an_adapter_s_rows_do_not_depend_on_the_batch_around_them(counts, rank, gated):
    """T_cap, the number of requests and of adapters stay; the order of the requests, the other ones' lengths, adapters and values change, so that
    the first one's rows lie elsewhere in other tiles, alone or beside others."""
    n, cap = counts[0], sum(counts) + 40
    ends = [150, 300] if gated else [256, 331]
    c = adapters.make(21, counts, cap, 2048, ends, rank, 5, ids=[3, 1, 0, 2], gated=gated)
    ctx = adapters.context()
    want = adapters.run(ctx, c, "silu")[:n]
    rng, g = np.random.default_rng(2), torch.Generator("cuda").manual_seed(3)
    for _ in range(6):
        lengths = rng.multinomial(cap - n, rng.dirichlet(np.ones(3)))
        order = rng.permutation(4)
        lens, ids = np.array([n, *lengths])[order], np.array([3, *rng.choice([-1, 0, 3, 4], 3)])[order]
        cu = np.concatenate([[0], np.cumsum(lens)])
        at = int(cu[list(order).index(0)])
        d = dict(c, ids=ids, hcu=cu, adapter=torch.tensor(ids, dtype=torch.int32, device="cuda"), cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        for name in ("x", "base"):
            t = torch.empty_strided(c[name].shape, c[name].stride(), dtype=c[name].dtype, device="cuda")
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
            t[at:at + n] = c[name][:n]
            d[name] = t
        assert torch.equal(adapters.run(ctx, d, "silu")[at:at + n], want)
