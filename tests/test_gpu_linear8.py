"""dcut_linear8 against its formula in 64 bits.

Tolerance: dcut_linear's (test_gpu_linear.py), whose sum is here that of a8 w8 (products of two e4m3 values are exact in fp32, the
sum is off by at most K 2^-23 sum |a8 w8|), times both scales: one rounding for the column's, one for the row's together with the bias, each 2^-24
of what it rounds, counted as 2^-23 (|z| + |bias|) and 2^-23 |z|.
"""
import numpy as np
import pytest
import torch

from tests.plain_reference import bf16_values, linear as plain
from tests.test_gpu_linear import NAN, SHAPES, context

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def values(t):
    return t.float().cpu().numpy().astype(np.float64)


def make(seed, T, cap, N, K, gated=False, bias=True, residual=False, scale=1.0):
    """Inputs as padded views; what no row or column of the product owns is NaN."""
    g = torch.Generator("cuda").manual_seed(seed)

    def rows8(rows):
        t = torch.full((rows + 1, -(-K // 16) * 16 + 16), NAN, device="cuda").to(F8)
        x = 60.0 * torch.randn((rows, K), generator=g, device="cuda") * torch.exp(torch.randn((rows, 1), generator=g, device="cuda"))
        t[:rows, :K] = x.clamp(-448, 448).to(F8)
        return t[:rows, :K]

    def scales(n, size):
        return size / 60 * torch.exp(2 * torch.rand(n, generator=g, device="cuda") - 1)

    vec = lambda: torch.randn(N, generator=g, device="cuda").to(torch.bfloat16)
    weight = lambda: (rows8(N), scales(N, K ** -0.5))
    res = None
    if residual:
        res = torch.full((cap + 1, -(-N // 8) * 8 + 8), NAN, dtype=torch.bfloat16, device="cuda")
        res[:T, :N] = torch.randn((T, N), generator=g, device="cuda").to(torch.bfloat16)
        res = res[:cap, :N]
    a_scale = scales(cap, scale)
    a_scale[T:] = NAN
    (w, ws), (w2, ws2) = weight(), weight() if gated else (None, None)
    return dict(a=rows8(cap), a_scale=a_scale, w=w, w_scale=ws, w2=w2, w2_scale=ws2, cu=torch.tensor([0, T // 2, T], dtype=torch.int32, device="cuda"),
                T=T, cap=cap, bias=vec() if bias else None, bias2=vec() if gated and bias else None, residual=res)


def run(ctx, c, act="none", **kw):
    return ctx.linear8(c["a"], c["a_scale"], c["w"], c["w_scale"], c["cu"], c["cap"], bias=c["bias"], act=act, w2=c["w2"], w2_scale=c["w2_scale"],
                       bias2=c["bias2"], residual=c["residual"], **kw)


def check(c, out, act="none", T=None, residual=None):
    T = c["T"] if T is None else T
    if not T:
        return
    f = lambda t: None if t is None else bf16_values(t)
    sa = values(c["a_scale"][:T])[:, None]
    a, bias, bias2 = values(c["a"][:T]) * sa, f(c["bias"]), f(c["bias2"])
    weight = lambda w, s: None if w is None else values(w) * values(s)[:, None]
    w, w2 = weight(c["w"], c["w_scale"]), weight(c["w2"], c["w2_scale"])
    res = f(c["residual"][:T]) if c["residual"] is not None else residual
    K = a.shape[1]
    want = plain(a, w, bias, act, w2, bias2, res)

    def pre(w_, b_):
        b_ = 0 if b_ is None else b_
        z = a @ w_.T
        return np.abs(z + b_), K * 2.0 ** -23 * (np.abs(a) @ np.abs(w_).T) + 2.0 ** -23 * (2 * np.abs(z) + np.abs(b_))

    _, e = pre(w, bias)
    y = np.abs(plain(a, w, bias, act))
    tol = 1.2 * e + 2.0 ** -14 * y + 1e-30
    if w2 is not None:
        u, eu = pre(w2, bias2)
        tol = tol * u + y * eu + tol * eu + 2.0 ** -22 * y * u
    tol += 2.0 ** -22 * np.abs(want) + (0 if res is None else 2.0 ** -23 * np.abs(res))
    tol = (1 + 2.0 ** -8) * tol + 2.0 ** -8 * np.abs(want)
    got = bf16_values(out[:T])
    assert np.isfinite(got).all()
    worst = (np.abs(got - want) / tol).max()
    assert worst <= 1, worst


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T,cap,N,K", SHAPES + [(77, 80, 300, 128), (77, 80, 300, 129), (200, 200, 500, 2176)])
def test_shapes(T, cap, N, K, gated):
    ctx, c = context(), make(T + N + K, T, cap, N, K, gated, residual=N % 2 == 1)
    out = torch.full((cap, N), 7.0, dtype=torch.bfloat16, device="cuda")
    run(ctx, c, "silu" if gated else "none", out=out)
    assert ctx.poll_device_status() == 0
    check(c, out, "silu" if gated else "none")
    assert (out[T:] == 7.0).all()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_epilogues(act, gated, bias, residual):
    for T in (5, 150):
        ctx, c = context(), make(11, T, T + 2, 203, 333, gated, bias, residual, scale=3.0)
        check(c, run(ctx, c, act), act)


@pytest.mark.parametrize("gated,plan", [(False, p) for p in (*range(7), *range(8, 15), *range(16, 23))] + [(True, p) for p in (0, 2, 4, 6, 8, 10, 12, 14)])
def test_every_plan(plan, gated, monkeypatch):
    """K above 1024 (512 counted in bf16 elements of a k-block), so that pairs and split K are open."""
    monkeypatch.setenv("DCUT_GEMM_FORCE", str(plan))
    ctx = context()
    for T, N, K in ((9, 331, 1200), (300, 331, 1100), (9, 336, 1300), (300, 336, 1200)):
        c = make(plan + T, T, T, N, K, gated, True, True)
        out = torch.full((T + 3, N), 7.0, dtype=torch.bfloat16, device="cuda")
        run(ctx, c, "gelu", out=out)
        assert ctx.poll_device_status() == 0
        check(c, out, "gelu")
        assert (out[T:] == 7.0).all()


def test_every_pair_of_8_bit_values():
    """One product per element of the output: all 256 x 256 pairs of codes, subnormals, zeros and NaN among them."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda")
    a = torch.zeros((256, 16), dtype=torch.uint8, device="cuda")
    a[:, 0] = codes
    one = torch.ones(256, device="cuda")
    a = a.view(F8)
    got = context().linear8(a, one, a.clone(), one, torch.tensor([0, 256], dtype=torch.int32, device="cuda"), 256)
    v = values(a[:, 0])
    want = torch.tensor(v[:, None] * v[None, :]).to(torch.bfloat16)                     # exact before the rounding
    assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want))


def test_long_sums_keep_small_terms():
    """A term 2^17 below the largest of its k-block, alone and many: the accumulator holds 32-bit values."""
    K, T = 4096, 8
    a, w = torch.zeros((T, K), device="cuda"), torch.zeros((16, K), device="cuda")
    w[:] = 1.0
    a[0, 0], a[0, 1] = 448.0, 2.0 ** -9
    a[1, 0], a[1, 1:] = 448.0, 2.0 ** -9
    a[2, 0], a[2, 2048], a[2, 1] = 448.0, -448.0, 2.0 ** -9
    one = torch.ones(16, device="cuda")
    out = context().linear8(a.to(F8), one[:T].contiguous(), w.to(F8), one, torch.tensor([0, T], dtype=torch.int32, device="cuda"), T,
                            residual=torch.full((T, 16), -448.0, dtype=torch.bfloat16, device="cuda"))
    got = out[:, 0].float().cpu()
    assert got[0] == 2.0 ** -9                                          # 448 + 2^-9 has 19 bits
    assert abs(float(got[1]) - 4095 * 2.0 ** -9) <= 2.0 ** -8 * 8       # so does every partial sum: exact up to the store
    assert got[2] == -448.0                                             # (448 - 448 + 2^-9) - 448, rounded to bf16


@pytest.mark.parametrize("ldo,shift", [(208, 0), (203, 0), (211, 3), (208, 1)])
def test_strided_out_and_in_place_residual(ldo, shift):
    T, N = 40, 203
    ctx, c = context(), make(5, T, T, N, 96)
    buf = torch.full((T * ldo + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[shift:shift + T * ldo].view(T, ldo)[:, :N]
    out.copy_(torch.randn((T, N), generator=torch.Generator("cuda").manual_seed(1), device="cuda"))
    before = bf16_values(out)
    c["residual"] = out
    run(ctx, c, "relu", out=out)
    c["residual"] = None
    check(c, out, "relu", residual=before)
    out.fill_(7.0)
    assert (buf == 7.0).all()                                          # nothing beside the rows


def test_nan_and_infinite_scales_stay_in_their_rows():
    T, N, K = 130, 96, 200
    ctx, c = context(), make(7, T, T, N, K, bias=True)
    want = run(ctx, c, "relu").clone()
    c["a"].view(torch.uint8)[4, 7] = 0x7f
    c["a_scale"][129] = NAN
    got = run(ctx, c, "relu")
    keep = [i for i in range(T) if i not in (4, 129)]
    assert torch.equal(got[keep], want[keep])
    assert torch.isnan(got[[4, 129]]).all()


def test_no_rows_and_too_many():
    ctx, c = context(), make(8, 20, 20, 50, 40)
    out = torch.full((24, 50), 7.0, dtype=torch.bfloat16, device="cuda")
    c["cu"][2] = 0
    run(ctx, c, out=out)
    assert ctx.poll_device_status() == 0 and (out == 7.0).all()
    c["cu"][2] = 23
    run(ctx, c, out=out)
    assert ctx.poll_device_status() == 10
    check(c, out)
    assert (out[20:] == 7.0).all()


def test_graph_replays_with_another_length_and_two_streams():
    ctx, c = context(), make(9, 200, 200, 300, 264, True, True, True)
    ctx2, c2 = context(), make(10, 60, 60, 1500, 2030)
    out, out2 = (torch.full((x["cap"], x["w"].shape[0]), 7.0, dtype=torch.bfloat16, device="cuda") for x in (c, c2))
    s, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run(ctx, c, "silu", out=out)
    for T in (200, 1, 131):
        c["cu"].copy_(torch.tensor([0, T // 2, T], dtype=torch.int32))
        out.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        with torch.cuda.stream(s2):
            run(ctx2, c2, out=out2)
        torch.cuda.synchronize()
        check(c, out, "silu", T=T)
        assert (out[T:] == 7.0).all()
        check(c2, out2)


def test_on_rows_that_the_norm_and_quantize_made():
    """The chain: norm to 8 bits, a weight quantised by rows, the product; and the values that were rounded, in bf16's place."""
    from paper_2607_14647_b200 import binding
    g = torch.Generator("cuda").manual_seed(12)
    T, N, K, ctx = 45, 200, 1000, context()
    x = torch.randn((T, K), generator=g, device="cuda").to(torch.bfloat16)
    w = (K ** -0.5 * torch.randn((N, K), generator=g, device="cuda")).to(torch.bfloat16)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    w8, ws = ctx.quantize(w, None, N)
    y8, s = binding.rows8(T, K), torch.empty(T, device="cuda")
    ctx.rms_norm(x, cu, T, out8=y8, scale8=s)
    out = ctx.linear8(y8, s, w8, ws, cu, T)
    check(dict(a=y8, a_scale=s, w=w8, w_scale=ws, w2=None, w2_scale=None, bias=None, bias2=None, residual=None, T=T), out)


def test_refusals_through_the_context():
    from paper_2607_14647_b200 import binding
    ctx, c = context(), make(12, 4, 4, 16, 24)
    with pytest.raises(KeyError):
        run(ctx, c, "tanh")
    with pytest.raises(binding.DcutError):
        ctx.linear8(c["a"].contiguous(), c["a_scale"], c["w"], c["w_scale"], c["cu"], 4)       # rows 24 elements apart
    with pytest.raises(AssertionError):
        ctx.linear8(c["a"].float(), c["a_scale"], c["w"], c["w_scale"], c["cu"], 4)
    with pytest.raises(AssertionError):
        ctx.linear8(c["a"], c["a_scale"][:3], c["w"], c["w_scale"], c["cu"], 4)


@pytest.mark.parametrize("T,cap,N,K", [(9700, 9700, 200, 1200), (100, 20000, 256, 1040)])
def test_very_many_rows_and_few_columns(T, cap, N, K):
    ctx, c = context(), make(16, T, cap, N, K)
    out = torch.full((cap, N), 7.0, dtype=torch.bfloat16, device="cuda")
    run(ctx, c, "relu", out=out)
    assert ctx.poll_device_status() == 0
    check(c, out, "relu")
    assert (out[T:] == 7.0).all()
