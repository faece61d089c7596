"""dcut_lora against its formula in 64 bits.

Tolerance.  s = x . a^T: an fp32 sum of K exact products, off by at most K 2^-23 sum |x a|; scaled (2^-24) and rounded to bf16 (2^-8 of it).
d: those errors times |b|, and an fp32 sum of rank exact products, rank 2^-23 sum |s b|.  base + d: 2^-24 of it.  The activation, the gate and the store
as in test_gpu_linear.py: slope below 1.2, 2^-14 of the value, both factors' errors, 2^-8 of the result.
"""
import numpy as np
import pytest
import torch

from tests.plain_reference import bf16_values, linear

pytestmark = pytest.mark.gpu
BF16, NAN = torch.bfloat16, float("nan")


def context():
    from paper_2607_14647_b200 import binding
    return binding.Context(max_B=8, max_gamma=4)


def make(seed, counts, cap, K, ends, rank, adapters, ids=None, gated=False, scale=True, pad=8, base_pad=0, start=0):
    """Packed requests of `counts` rows from row `start` on; rows that nobody owns are NaN, and so is what lies beside the rows."""
    g = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    counts = np.asarray(counts)
    cu = start + np.concatenate([[0], np.cumsum(counts)])
    T, N, kp, sr = int(cu[-1]), ends[-1], -(-K // 8) * 8 + pad, len(ends) * rank
    if ids is None:
        ids = rng.integers(-1, adapters, len(counts))

    def rows(cols, extra):
        t = torch.full((cap + 1, cols + extra), NAN, dtype=BF16, device="cuda")
        t[start:T, :cols] = n(T - start, cols).to(BF16)
        return t[:cap, :cols]

    a = torch.full((adapters + 1, sr, kp), NAN, dtype=BF16, device="cuda")
    a[:adapters, :, :K] = (K ** -0.5 * n(adapters, sr, K)).to(BF16)
    b = torch.full((adapters + 1, N, rank), NAN, dtype=BF16, device="cuda")
    b[:adapters] = n(adapters, N, rank).to(BF16)
    i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    return dict(x=rows(K, -K % 8 + pad), a=a[:adapters, :, :K], b=b[:adapters], base=rows(N, base_pad), ids=np.asarray(ids), adapter=i32(ids), cu=i32(cu), cap=cap,
                scale=(0.5 + torch.rand(adapters, generator=g, device="cuda")) if scale else None, ends=list(ends), gated=gated, hcu=cu,
                width=N // 2 if gated else N)


def run(ctx, c, act="none", out=None, pad=0):
    if out is None:
        out = torch.full((c["cap"] + 1, c["width"] + pad), 7.0, dtype=BF16, device="cuda")
    ctx.lora(c["x"], c["a"], c["b"], c["adapter"], c["base"], c["cu"], c["cap"], out=out[:, :c["width"]], scale=c["scale"], slices=c["ends"], act=act, gated=c["gated"])
    return out


def expected(c, act="none", base=None, s_rounding=2.0 ** -8, parts=1):
    """(want, tolerance) of the rows that requests own."""
    N, ends, r = c["ends"][-1], c["ends"], c["b"].shape[2]
    lo, hi = int(c["hcu"][0]), int(c["hcu"][-1])
    x, base = bf16_values(c["x"]), bf16_values(c["base"]) if base is None else base
    z, e = base[lo:hi].copy(), np.zeros((hi - lo, N))
    for i, t in enumerate(c["ids"]):
        p, q = int(c["hcu"][i]), int(c["hcu"][i + 1])
        if t < 0 or p == q:
            continue
        a, b = bf16_values(c["a"][t]), bf16_values(c["b"][t])
        f = 1.0 if c["scale"] is None else float(c["scale"][t])
        K = a.shape[1]
        s, es = f * (x[p:q] @ a.T), f * K * 2.0 ** -23 * (np.abs(x[p:q]) @ np.abs(a).T)
        es = es * (1 + 2.0 ** -7) + (s_rounding + 2.0 ** -24) * np.abs(s)
        first = 0
        for j, end in enumerate(ends):
            k, n = slice(j * r, (j + 1) * r), slice(first, end)
            z[p - lo:q - lo, n] += s[:, k] @ b[n].T
            e[p - lo:q - lo, n] = es[:, k] @ np.abs(b[n]).T + parts * r * 2.0 ** -23 * 1.01 * (np.abs(s[:, k]) @ np.abs(b[n]).T)
            first = end
    e += 2.0 ** -24 * np.abs(z)
    one = np.eye(1)

    def activated(v):
        return linear(v.reshape(-1, 1), one, act=act).reshape(v.shape)

    if c["gated"]:
        zg, zu, eg, eu = z[:, :N // 2], z[:, N // 2:], e[:, :N // 2], e[:, N // 2:]
        y = activated(zg)
        want = y * zu
        ey = 1.2 * eg + 2.0 ** -14 * np.abs(y) + 1e-30
        tol = ey * np.abs(zu) + np.abs(y) * eu + ey * eu + 2.0 ** -22 * np.abs(want)
    else:
        want = activated(z)
        tol = (1.2 * e + 2.0 ** -14 * np.abs(want) + 1e-30) if act != "none" else e
    return want, (1 + 2.0 ** -8) * tol + 2.0 ** -8 * np.abs(want) + 1e-38


def check(c, out, act="none", base=None, untouched=True):
    lo, hi = int(c["hcu"][0]), int(c["hcu"][-1])
    want, tol = expected(c, act, base)
    got = bf16_values(out)[lo:hi, :c["width"]]
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    if untouched:
        assert (out[:lo] == 7).all() and (out[hi:] == 7).all() and (out[:, c["width"]:] == 7).all()


RAGGED = [1, 17, 0, 3, 40, 16, 33, 1]


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 96, 128])
@pytest.mark.parametrize("counts", [[1], [1] * 5, RAGGED, [150, 1, 64]])
def test_ranks_and_row_counts(rank, counts):
    for ends in ([200], [96, 131]):
        c = make(rank + len(counts), counts, sum(counts) + 3, 300, ends, rank, 3)
        ctx = context()
        check(c, run(ctx, c))
        assert ctx.poll_device_status() == 0


@pytest.mark.parametrize("K", [1, 7, 8, 31, 32, 33, 63, 255, 256, 257, 1000, 2048, 4100])
@pytest.mark.parametrize("ends", [[1], [40], [33, 34], [8, 72, 80], [31, 95, 96, 200], [1500]])
def test_sizes(K, ends):
    c = make(K + ends[-1], [2, 1, 19], 24, K, ends, 16, 2, ids=[1, 0, 1])
    check(c, run(context(), c))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("counts", [[1, 3], RAGGED, [100, 70]])
def test_activations_and_gate(act, gated, counts):
    for ends in ([300], [150, 300], [13, 26] if gated else [13, 27]):
        for rank in (16, 32):
            c = make(len(act) + rank, counts, sum(counts) + 1, 200, ends, rank, 4, gated=gated)
            check(c, run(context(), c, act), act)


@pytest.mark.parametrize("base_pad,pad", [(0, 0), (3, 0), (8, 8), (1, 5), (0, 3)])
def test_strides(base_pad, pad):
    for ends in ([64, 200], [203]):
        c = make(base_pad, RAGGED, sum(RAGGED), 100, ends, 16, 3, base_pad=base_pad)
        check(c, run(context(), c, pad=pad))


def test_odd_places_of_base_and_out():
    c = make(4, [5, 9], 14, 64, [77], 16, 2)
    for shift in (1, 3, 8):
        buf = torch.full((16 * 80 + 8,), 7.0, dtype=BF16, device="cuda")
        base = torch.zeros(14 * 80 + 8, dtype=BF16, device="cuda")[shift:shift + 14 * 80].view(14, 80)[:, :77]
        base.copy_(c["base"])
        out = buf[shift:shift + 15 * 80].view(15, 80)
        check(c, run(context(), dict(c, base=base), out=out))


@pytest.mark.parametrize("counts", [[1, 1, 1], RAGGED, [100, 90]])
def test_in_place_leaves_rows_without_an_adapter_alone(counts):
    ids = [i % 3 - 1 for i in range(len(counts))]
    c = make(5, counts, sum(counts) + 2, 128, [64, 160], 16, 2, ids=ids)
    before = c["base"].clone()
    ctx = context()
    ctx.lora(c["x"], c["a"], c["b"], c["adapter"], c["base"], c["cu"], c["cap"], out=c["base"], scale=c["scale"], slices=c["ends"])
    check(c, c["base"], base=bf16_values(before), untouched=False)
    for i, t in enumerate(ids):
        if t < 0:
            rows = slice(int(c["hcu"][i]), int(c["hcu"][i + 1]))
            assert torch.equal(c["base"][rows], before[rows])
    # with an activation in place, every row is activated
    c["base"].copy_(before)
    ctx.lora(c["x"], c["a"], c["b"], c["adapter"], c["base"], c["cu"], c["cap"], out=c["base"], scale=c["scale"], slices=c["ends"], act="relu")
    check(c, c["base"], "relu", base=bf16_values(before), untouched=False)


@pytest.mark.parametrize("ids", [[-1, -1, -1], [-7, 2, -1], [2, 2, 2]])
@pytest.mark.parametrize("scale", [False, True])
def test_none_some_and_one_for_all(ids, scale):
    c = make(6, [4, 20, 1], 30, 96, [100], 16, 3, ids=ids, scale=scale)
    out = run(context(), c)
    check(c, out)
    if max(ids) < 0:
        assert torch.equal(out[:25], c["base"][:25])


def test_rows_ahead_of_the_first_request_and_empty_requests():
    c = make(7, [0, 5, 0, 0, 2, 0], 15, 64, [72], 16, 2, start=4)
    check(c, run(context(), c))
    c = make(8, [0, 0], 3, 64, [72], 16, 2)
    assert (run(context(), c) == 7).all()


@pytest.mark.parametrize("B", [255, 256, 257, 700, 3000])
def test_many_requests(B):
    counts = np.random.default_rng(B).integers(0, 4, B)
    c = make(B, counts, int(counts.sum()) + 5, 72, [48], 8, 5)
    check(c, run(context(), c))


@pytest.mark.parametrize("n_slices,rank", [(1, 256), (2, 128), (4, 64), (3, 80)])
def test_the_most_ranks(n_slices, rank):
    ends = [50 * (i + 1) for i in range(n_slices)]
    for counts in ([1], [17, 20], [130]):
        c = make(rank, counts, sum(counts), 520, ends, rank, 2, ids=[i % 2 for i in range(len(counts))])
        check(c, run(context(), c))


@pytest.mark.parametrize("counts,rank,n_slices", [([9000], 256, 1), ([5000, 0, 4100], 64, 4), ([1] * 8000, 8, 1)])
def test_more_rows_than_the_scratch_holds_at_a_time(counts, rank, n_slices):
    c = make(rank, counts, sum(counts) + 2, 64, [24 * (i + 1) for i in range(n_slices)], rank, 2, ids=[i % 2 for i in range(len(counts))])
    ctx = context()
    check(c, run(ctx, c))
    assert ctx.poll_device_status() == 0


def test_an_adapter_that_does_not_exist_and_a_packing_above_the_cap():
    ctx, c = context(), make(9, [2, 3, 4], 9, 64, [40], 16, 3, ids=[0, 1, 2])
    c["adapter"][1] = 3
    out = run(ctx, c)
    assert ctx.poll_device_status() == 11
    check(dict(c, ids=np.array([0, -1, 2])), out)
    for base in (c["base"], c["base"].clone()):                         # also where such a request has no tile
        ctx.lora(c["x"], c["a"], c["b"], c["adapter"], base, c["cu"], 9, out=base)
        assert ctx.poll_device_status() == 11
    c = make(10, [2, 3, 4], 9, 64, [40], 16, 3, ids=[0, 1, 2])
    out = torch.full((10, 40), 7.0, dtype=BF16, device="cuda")
    ctx.lora(c["x"], c["a"], c["b"], c["adapter"], c["base"], c["cu"], 7, out=out, scale=c["scale"])
    assert ctx.poll_device_status() == 10
    assert (out[7:] == 7).all()
    c["hcu"] = np.array([0, 2, 5, 7])
    check(c, out)
    many = make(11, [1] * 600, 600, 32, [16], 8, 2)
    many["adapter"][599] = 2
    run(ctx, many)
    assert ctx.poll_device_status() == 11


def test_infinities_and_nan_stay_in_their_rows():
    c = make(12, [3, 20, 1], 24, 128, [64, 128], 24, 2, ids=[0, 1, 0])
    ctx = context()
    want = run(ctx, c)
    c["x"][1, 5], c["x"][10, 127], c["base"][23, 70] = NAN, float("inf"), NAN
    got = run(ctx, c)
    keep = [r for r in range(24) if r not in (1, 10, 23)]
    assert torch.equal(got[keep], want[keep])
    assert torch.isnan(got[1]).all() and not torch.isfinite(got[10].float()).any()
    assert torch.isnan(got[23, 70]) and torch.equal(got[23, :70], want[23, :70]) and torch.equal(got[23, 71:], want[23, 71:])


def test_a_slice_of_infinite_weights_stays_in_its_columns():
    c = make(13, [4], 4, 64, [40, 80], 8, 1, ids=[0])
    ctx = context()
    want = run(ctx, c)
    c["a"][0, 8:] = float("inf")                                          # the second slice's
    got = run(ctx, c)
    assert torch.equal(got[:4, :40], want[:4, :40]) and not torch.isfinite(got[:4, 40:].float()).any()


def test_repeated_calls_are_bit_identical_whatever_else_is_in_the_batch():
    ctx, c = context(), make(14, [9, 17, 5], 31, 2048, [512, 640], 16, 3, ids=[0, 1, 2])
    first = run(ctx, c)
    for _ in range(20):
        assert torch.equal(run(ctx, c), first)


def test_graph_replays_with_other_requests_and_two_streams():
    ctx, c = context(), make(15, [17, 3, 9, 4], 60, 512, [256], 32, 4, ids=[0, 1, 2, 3])
    ctx2, c2 = context(), make(16, [40, 50], 90, 1000, [300, 600], 16, 2, ids=[1, 0], gated=True)
    out, out2 = (torch.full((x["cap"] + 1, x["width"]), 7.0, dtype=BF16, device="cuda") for x in (c, c2))
    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run(ctx, c, out=out)
    for ids, counts in (([0, 1, 2, 3], [17, 3, 9, 4]), ([3, 3, -1, 0], [1, 1, 1, 1]), ([-1, 2, 1, 0], [0, 9, 17, 2])):
        c["ids"], c["hcu"] = np.array(ids), np.concatenate([[0], np.cumsum(counts)])
        c["adapter"].copy_(torch.tensor(ids, dtype=torch.int32))
        c["cu"].copy_(torch.tensor(c["hcu"], dtype=torch.int32))
        T = int(c["hcu"][-1])
        for n in ("x", "base"):
            c[n][:T] = torch.randn(c[n][:T].shape, device="cuda").to(BF16)
        out.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        with torch.cuda.stream(s2):
            run(ctx2, c2, "silu", out=out2)
        torch.cuda.synchronize()
        check(c, out)
        check(c2, out2, "silu")


def test_adapters_and_rows_behind_2_31_elements():
    g = torch.Generator("cuda").manual_seed(17)
    m, N, rank, K, T = 700, 100000, 32, 64, 3
    b = torch.zeros((m, N, rank), dtype=BF16, device="cuda")
    b[-1] = torch.randn((N, rank), generator=g, device="cuda").to(BF16)
    c = make(17, [T], T, K, [N], rank, 1, ids=[0])
    a = torch.zeros((m, rank, K), dtype=BF16, device="cuda")
    a[-1] = c["a"][0]
    c["b"] = b[-1:]
    out = torch.full((T, N), 7.0, dtype=BF16, device="cuda")
    ids = torch.tensor([m - 1], dtype=torch.int32, device="cuda")
    context().lora(c["x"], a, b, ids, c["base"], c["cu"], T, out=out)
    check(dict(c, scale=None), out)
    del b
    ld, T = 2 << 20, 1100
    c = make(18, [1, T - 1], T, 64, [40], 16, 2, ids=[0, 1])
    base = torch.empty((T, ld), dtype=BF16, device="cuda")[:, :40]
    base.copy_(c["base"])
    out = torch.empty((T, ld), dtype=BF16, device="cuda")[:, :40]
    check(dict(c, base=base), run(context(), dict(c, base=base), out=out), untouched=False)


def test_refusals_through_the_context():
    ctx, c = context(), make(19, [2, 3], 5, 64, [40], 16, 3)
    kw = dict(out=None)
    for change in (dict(a=c["a"].float()), dict(b=c["b"][:, :39]), dict(a=c["a"][:, :8]), dict(adapter=c["adapter"][:1]), dict(base=c["base"][:4]), dict(x=c["x"].cpu())):
        with pytest.raises(AssertionError):
            ctx.lora(*(dict(c, **change)[n] for n in ("x", "a", "b", "adapter", "base", "cu", "cap")), **kw)
    with pytest.raises(AssertionError):
        ctx.lora(c["x"], c["a"], c["b"], c["adapter"], c["base"], c["cu"], 5, slices=[20, 39])
    with pytest.raises(KeyError):
        ctx.lora(c["x"], c["a"], c["b"], c["adapter"], c["base"], c["cu"], 5, act="tanh")


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 64, 96])
@pytest.mark.parametrize("counts,gated", [([1], False), (RAGGED, False), ([150, 64], False), ([150, 64], True)])
def test_the_low_rank_product_keeps_16_bits(rank, counts, gated):
    """s enters the second product as two bf16 values: the first is off by half a step, at most 2^(e-8) where |s| is in [2^e, 2^(e+1)); that rest lies
    in a binade no higher than 2^(e-9) (2^(e-8) itself is exact), so its rounding is off by 2^(e-17) at most: 2^-17 |s|.  No base, so that sums
    that cancel show it: without the low parts this term would be 2^9 times as large.  The second sum has twice the rank's terms."""
    c = make(1000 + rank, counts, sum(counts) + 1, 64, [80, 160] if gated else [96, 200], rank, 3, ids=[i % 3 for i in range(len(counts))], gated=gated)
    c["base"].zero_()
    lo, hi = int(c["hcu"][0]), int(c["hcu"][-1])
    want, tol = expected(c, "none", s_rounding=2.0 ** -17, parts=2)
    got = bf16_values(run(context(), c))[lo:hi, :c["width"]]
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    # the same sums from one bf16 value would not pass (formed here, in 64 bits, where nothing follows the sum)
    if gated or sum(counts) < 100:
        return
    x, z = bf16_values(c["x"])[lo:hi], np.zeros_like(want)
    for i, t in enumerate(c["ids"]):
        rows = slice(int(c["hcu"][i]) - lo, int(c["hcu"][i + 1]) - lo)
        if t >= 0:
            f = 1.0 if c["scale"] is None else float(c["scale"][t])
            s = bf16_values(torch.from_numpy(f * (x[rows] @ bf16_values(c["a"][t]).T)).to(torch.bfloat16))
            first = 0
            for j, end in enumerate(c["ends"]):
                z[rows, first:end] = s[:, j * rank:(j + 1) * rank] @ bf16_values(c["b"][t])[first:end].T
                first = end
    assert (np.abs(z - want) > tol).any()
