"""dcut_lora on small whole numbers, where every sum is exact and the result is the formula's, rounded once: nothing of the low-rank product may be
lost, wherever it lies in its two bf16 parts.

x and a are whole numbers up to 4, so s = x . a^T has some 8 to 12 bits (all here are checked: below 2^15): two bf16 values hold them (16 bits), one does
not (8; the last test); b and base are whole numbers, and every sum stays below 2^24.  The gate's product is one fp32 multiplication.  So no tolerance."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def context():
    from paper_2607_14647_b200 import binding
    return binding.Context(max_B=8, max_gamma=4)


def make(seed, counts, K, ends, rank, adapters=3, ids=None, pad=0):
    rng = np.random.default_rng(seed)
    T, N = int(np.sum(counts)), ends[-1]
    whole = lambda most, *s: rng.integers(-most, most + 1, s).astype(np.float64)
    return dict(x=whole(4, T, K), a=whole(4, adapters, len(ends) * rank, K), b=whole(4, adapters, N, rank), base=whole(100, T, N), scale=2.0 ** rng.integers(-1, 3, adapters),
                ids=np.asarray([i % (adapters + 1) - 1 for i in range(len(counts), 0, -1)] if ids is None else ids), counts=np.asarray(counts), ends=list(ends), pad=pad)


def rows(v, pad):
    """A view of rows that start on 16 bytes and lie `pad` elements further apart."""
    t = torch.full((v.shape[0] + 1, -(-v.shape[1] // 8) * 8 + pad), float("nan"), dtype=BF16, device="cuda")
    t[:v.shape[0], :v.shape[1]] = torch.from_numpy(v).to(BF16)
    return t[:v.shape[0], :v.shape[1]]


def run(ctx, c, act="none", gated=False, in_place=False):
    m, sr, K = c["a"].shape
    T, N, pad = c["base"].shape[0], c["ends"][-1], c["pad"]
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    a = rows(c["a"].reshape(m * sr, K), 8)
    a = a.as_strided((m, sr, K), (sr * a.stride(0), a.stride(0), 1))
    base = torch.full((T, N + pad), 7.0, dtype=BF16, device="cuda")[:, :N]
    base.copy_(torch.from_numpy(c["base"]))
    out = base if in_place else torch.full((T, (N // 2 if gated else N) + pad), 7.0, dtype=BF16, device="cuda")[:, :N // 2 if gated else N]
    ctx.lora(rows(c["x"], 8), a, torch.from_numpy(c["b"]).to(BF16).cuda(), i32(c["ids"]), base, i32(np.concatenate([[0], np.cumsum(c["counts"])])), T, out=out,
             scale=torch.from_numpy(c["scale"]).float().cuda(), slices=c["ends"], act=act, gated=gated)
    assert ctx.poll_device_status() == 0
    return out


def expected(c, act="none", gated=False, held=lambda s: s):
    z, row = c["base"].copy(), 0
    rank = c["b"].shape[2]
    for t, n in zip(c["ids"], c["counts"]):
        if t >= 0 and n:
            s, lo = c["scale"][t] * (c["x"][row:row + n] @ c["a"][t].T), 0
            assert np.abs(s).max() < 2 ** 15
            s = held(s)
            for j, hi in enumerate(c["ends"]):
                z[row:row + n, lo:hi] += s[:, j * rank:(j + 1) * rank] @ c["b"][t, lo:hi].T
                lo = hi
        row += n
    assert np.abs(z).max() < 2 ** 22                                     # (halves among them: 23 bits)
    f = np.maximum(z, 0) if act == "relu" else z
    if gated:
        half = c["ends"][-1] // 2
        f = f[:, :half].astype(np.float32) * z[:, half:].astype(np.float32)
    return torch.from_numpy(np.ascontiguousarray(f)).float().to(BF16)


def check(c, act="none", gated=False, in_place=False):
    want = expected(c, act, gated)
    got = run(context(), c, act, gated, in_place).cpu()
    assert torch.equal(got + 0.0, want + 0.0), f"{int((got != want).sum())} of {want.numel()} differ"       # (-0 is 0)


COUNTS = [[1], [1] * 7, [1, 17, 0, 3, 40, 16, 33, 1], [150, 1, 64], [300, 310]]


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 48, 56, 64, 80, 96, 112, 128, 256])
@pytest.mark.parametrize("counts", COUNTS)
def test_ranks(rank, counts):
    for ends in ([200],) if rank > 128 else ([200], [96, 131]):
        check(make(rank + len(counts), counts, 1000, ends, rank, ids=[i % 3 for i in range(len(counts))]))


@pytest.mark.parametrize("rank", [8, 24, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("act", ["none", "relu"])
def test_gated(rank, counts, act):
    for ends in ([300], [150, 300], [13, 26]):
        if len(ends) * rank <= 256:
            check(make(rank, counts, 500, ends, rank, ids=[2 - i % 3 for i in range(len(counts))]), act, gated=True)


@pytest.mark.parametrize("K", [600, 1003, 2048, 4100, 12288])
@pytest.mark.parametrize("ends", [[1], [40], [33, 34], [8, 72, 80], [31, 95, 96, 200], [1500]])
def test_sizes(K, ends):
    for counts in ([2, 1, 19], [1], [70, 60]):
        check(make(K + ends[-1], counts, K, ends, 16, ids=[2, 0, 2][:len(counts)]))


@pytest.mark.parametrize("K", [1, 7, 63, 64, 65])
def test_short_sums(K):
    check(make(K, [5, 30, 1], K, [90], 24))


@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("counts", COUNTS[2:])
def test_strides_rows_without_an_adapter_and_in_place(pad, counts):
    for act in ("none", "relu"):
        for in_place in (False, True):
            check(make(pad, counts, 800, [64, 203], 32, ids=[i % 4 - 1 for i in range(len(counts), 0, -1)], pad=pad), act, in_place=in_place)


def test_more_rows_than_the_scratch_holds_and_more_requests_than_are_grouped():
    check(make(5, [9000], 600, [24], 256, adapters=1, ids=[0]))
    counts = np.random.default_rng(1).integers(0, 4, 700)
    check(make(6, counts, 600, [48], 8, adapters=5, ids=[i % 6 - 1 for i in range(700)]))


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("gated", [False, True])
def test_one_bf16_value_would_not_do(rank, gated):
    """(The oracle alone: the cases above tell the two apart.)"""
    c = make(rank, COUNTS[2], 4100, [150, 300], rank)
    one = expected(c, "none", gated, lambda s: torch.from_numpy(s).to(BF16).double().numpy())
    assert (one != expected(c, "none", gated)).any()
