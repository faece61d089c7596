"""dcut_linear against its formula in 64 bits.

Tolerance.  z, an fp32 sum of K exact products: off by at most E = K 2^-23 sum |a w|; the bias adds a rounding, 2^-23 (|z| +
|bias|).  An activation has a slope below 1.2 and is evaluated to 2^-14 of its value: the exponential to 2 + 1.2 |x| units of
2^-23, the complementary error function to 2 x^2 of those through its rounded argument, both below 2^-14 where the value is
above 1e-30.  The gate's product takes both factors' errors.  The residual adds 2^-23 of the sum, the store 2^-8 of the
result (half a step of bf16).
"""
import numpy as np
import pytest
import torch

from tests.plain_reference import bf16_values, linear as plain

pytestmark = pytest.mark.gpu
NAN = float("nan")


def ceil8(n):
    return -(-n // 8) * 8


def context():
    from paper_2607_14647_b200 import binding
    return binding.Context(max_B=8, max_gamma=4, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_req=4)


def make(seed, T, cap, N, K, gated=False, bias=True, residual=False, scale=1.0):
    """Inputs as padded views; what no row or column of the product owns is NaN."""
    g = torch.Generator("cuda").manual_seed(seed)

    def view(rows, cols, live=None, s=1.0, pad=1):
        t = torch.full((rows + pad, ceil8(cols) + 8), NAN, dtype=torch.bfloat16, device="cuda")
        t[:rows if live is None else live, :cols] = (s * torch.randn((rows if live is None else live, cols), generator=g, device="cuda")).to(torch.bfloat16)
        return t[:rows, :cols]

    vec = lambda: torch.randn(N, generator=g, device="cuda").to(torch.bfloat16)
    c = dict(a=view(cap, K, T, scale), w=view(N, K, s=K ** -0.5), cu=torch.tensor([0, T // 2, T], dtype=torch.int32, device="cuda"), T=T, cap=cap,
             bias=vec() if bias else None, w2=view(N, K, s=K ** -0.5) if gated else None, bias2=vec() if gated and bias else None,
             residual=view(cap, N, T) if residual else None)
    return c


def run(ctx, c, act="none", **kw):
    return ctx.linear(c["a"], c["w"], c["cu"], c["cap"], bias=c["bias"], act=act, w2=c["w2"], bias2=c["bias2"], residual=c["residual"], **kw)


def check(c, out, act="none", T=None, residual=None):
    T = c["T"] if T is None else T
    if not T:
        return
    f = lambda t: None if t is None else bf16_values(t)
    a, w, w2, bias, bias2 = f(c["a"][:T]), f(c["w"]), f(c["w2"]), f(c["bias"]), f(c["bias2"])
    res = f(c["residual"][:T]) if c["residual"] is not None else residual
    K = a.shape[1]
    want = plain(a, w, bias, act, w2, bias2, res)

    def pre(w_, b_):
        b_ = 0 if b_ is None else b_
        z = a @ w_.T
        return np.abs(z + b_), K * 2.0 ** -23 * (np.abs(a) @ np.abs(w_).T) + 2.0 ** -23 * (np.abs(z) + np.abs(b_))

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


SHAPES = [(1, 1, 1, 1), (1, 16, 8, 17), (3, 3, 4096, 64), (7, 16, 6144, 4096), (33, 64, 31, 8), (64, 64, 257, 129), (65, 65, 130, 65),
          (128, 200, 9000, 127), (129, 129, 256, 2048), (255, 300, 96, 1003), (257, 257, 2051, 191), (333, 512, 12000, 100), (640, 640, 2048, 512),
          (1000, 1088, 1025, 77)]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("T,cap,N,K", SHAPES)
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
@pytest.mark.parametrize("T", [5, 150])
def test_epilogues(T, act, gated, bias, residual):
    ctx, c = context(), make(11, T, T + 2, 203, 333, gated, bias, residual, scale=3.0)
    check(c, run(ctx, c, act), act)


@pytest.mark.parametrize("plan", ["0", "6", "2", "8", "12", "14", "16", "20", "22"])
@pytest.mark.parametrize("gated", [False, True])
def test_every_way_of_running(plan, gated, monkeypatch):
    monkeypatch.setenv("DCUT_GEMM_FORCE", plan)                       # (a plan that a launch cannot take falls back to the rule)
    ctx = context()
    for T, N, K in ((9, 331, 200), (200, 777, 520)):
        c = make(int(plan) + T, T, T, N, K, gated, True, True)
        check(c, run(ctx, c, "gelu"), "gelu")


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_activation_range(act):
    """z itself from -12 to 12 and far beyond: no cancellation in the tails, no overflow."""
    z = np.concatenate([np.linspace(-12, 12, 700), np.float32([-1e30, -3e4, -100.0, -40.0, 0.0, 40.0, 100.0, 3e4, 1e30])])
    a = torch.tensor(z, dtype=torch.float32, device="cuda").to(torch.bfloat16)[:, None].expand(-1, 8).clone()
    a[:, 1:] = 0
    w = torch.zeros((8, 8), dtype=torch.bfloat16, device="cuda")
    w[:, 0] = 1.0
    c = dict(a=a, w=w, cu=torch.tensor([0, len(z)], dtype=torch.int32, device="cuda"), T=len(z), cap=len(z), bias=None, w2=None, bias2=None, residual=None)
    check(c, run(context(), c, act), act)


@pytest.mark.parametrize("ldo,shift", [(208, 0), (203, 0), (211, 3), (208, 1)])
def test_strided_out_and_in_place_residual(ldo, shift):
    T, N = 40, 203
    ctx, c = context(), make(5, T, T, N, 96)
    buf = torch.full((T * ldo + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[shift:shift + T * ldo].view(T, ldo)[:, :N]
    g = torch.Generator("cuda").manual_seed(1)
    out.copy_(torch.randn((T, N), generator=g, device="cuda"))
    before = bf16_values(out)
    ctx.linear(c["a"], c["w"], c["cu"], T, out=out, bias=c["bias"], act="relu", residual=out)
    check(c, out, "relu", residual=before)
    out.fill_(7.0)
    assert (buf == 7.0).all()                                          # nothing beside the rows


def test_bias_and_weights_at_odd_places():
    T, N, K = 20, 77, 64
    ctx, c = context(), make(6, T, T, N, K, True, True, True)
    for n in ("bias", "bias2"):
        b = torch.full((N + 4,), NAN, dtype=torch.bfloat16, device="cuda")
        b[3:3 + N] = c[n]
        c[n] = b[3:3 + N]
    check(c, run(ctx, c, "silu"), "silu")


def test_infinities_and_nan_stay_in_their_rows():
    T, N, K = 130, 96, 200
    ctx, c = context(), make(7, T, T, N, K, bias=True)
    want = run(ctx, c, "relu").clone()
    c["a"][4, 7], c["a"][129, 199] = NAN, float("inf")
    got = run(ctx, c, "relu")
    keep = [i for i in range(T) if i not in (4, 129)]
    assert torch.equal(got[keep], want[keep])
    assert torch.isnan(got[4]).all()


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
    assert ctx.poll_device_status() == 0


def test_graph_replays_with_another_length_and_two_streams():
    ctx, c = context(), make(9, 200, 200, 300, 264, True, True, True)
    ctx2, c2 = context(), make(10, 60, 60, 1500, 1030)
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


def test_refusals_through_the_context():
    from paper_2607_14647_b200 import binding
    ctx, c = context(), make(12, 4, 4, 16, 24)
    with pytest.raises(KeyError):
        run(ctx, c, "tanh")
    with pytest.raises(binding.DcutError):
        ctx.linear(c["a"][:, :21].contiguous(), c["w"][:, :21], c["cu"], 4)       # rows 21 elements apart
    with pytest.raises(AssertionError):
        ctx.linear(c["a"].float(), c["w"], c["cu"], 4)


@pytest.mark.parametrize("N,ld", [(40, 2000008), (37, 2000003)])
def test_rows_behind_two_to_the_31_elements(N, ld):
    T = 1100
    ctx, c = context(), make(13, T, T, N, 72)
    out, residual = (torch.empty((T, ld), dtype=torch.bfloat16, device="cuda")[:, :N] for _ in "or")
    residual.copy_(make(14, T, T, N, 8, residual=True)["residual"])
    c["residual"] = residual
    run(ctx, c, "relu", out=out)
    check(c, out, "relu")


def test_tensors_of_another_device_are_refused(monkeypatch):
    ctx, c = context(), make(15, 4, 4, 16, 24)
    out = run(ctx, c)
    with pytest.raises(AssertionError):
        run(ctx, dict(c, bias=c["bias"].cpu()))
    with pytest.raises(AssertionError):
        run(ctx, c, out=out.cpu())
    monkeypatch.setattr(ctx, "device", 1)                      # as if the context lived on the next GPU
    with pytest.raises(AssertionError):
        run(ctx, c)


@pytest.mark.parametrize("T,cap,N,K", [(9700, 9700, 200, 600), (12345, 13000, 64, 1000), (9217, 9300, 33, 640), (100, 20000, 256, 520)])
def test_very_many_rows_and_few_columns(T, cap, N, K):
    """More row blocks than the table of plans has entries, where a single wave of pairs would do for that many and no more."""
    ctx, c = context(), make(16, T, cap, N, K)
    out = torch.full((cap, N), 7.0, dtype=torch.bfloat16, device="cuda")
    run(ctx, c, "relu", out=out)
    assert ctx.poll_device_status() == 0
    check(c, out, "relu")
    assert (out[T:] == 7.0).all()


def test_very_many_rows_of_the_layer_s_product():
    from paper_2607_14647_b200 import binding
    ctx = binding.Context(max_B=8192, max_gamma=1, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_req=4)
    T, N, K = 9700, 256, 640
    c = make(17, T, T, N, K, bias=False, residual=True)
    a, w, res = (c[n].contiguous() for n in ("a", "w", "residual"))
    out = torch.full((T, N), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.gemm_bf16(a, w, torch.tensor([0, T], dtype=torch.int32, device="cuda"), T, out, mode=1, residual=res)
    torch.cuda.synchronize()
    check(c, out)


@pytest.mark.parametrize("gated,plan", [(False, p) for p in (*range(7), *range(8, 15), *range(16, 23))] + [(True, p) for p in (0, 2, 4, 6, 8, 10, 12, 14)])
def test_every_plan_at_lengths_that_can_take_it(plan, gated, monkeypatch):
    """K above 512, so that pairs and split K are open (tests/test_gemm_plan.py holds that these launches do take the plan): the
    half activation box, one and two pair tiles of rows, odd N (2-byte rows and residual); even N (vectors)."""
    monkeypatch.setenv("DCUT_GEMM_FORCE", str(plan))
    ctx = context()
    for T, N, K in ((9, 331, 584), (300, 331, 600), (9, 336, 584), (300, 336, 600)):
        c = make(plan + T, T, T, N, K, gated, True, True)
        out = torch.full((T + 3, N), 7.0, dtype=torch.bfloat16, device="cuda")
        run(ctx, c, "gelu", out=out)
        assert ctx.poll_device_status() == 0
        check(c, out, "gelu")
        assert (out[T:] == 7.0).all()


@pytest.mark.parametrize("gated", [False, True])
def test_few_k_blocks_whatever_is_forced(gated, monkeypatch):
    """Up to K = 512 the pair modes are closed: a forced one falls back to the rule."""
    monkeypatch.setenv("DCUT_GEMM_FORCE", "8")
    ctx = context()
    for T, N, K in ((9, 331, 512), (300, 331, 64)):
        c = make(18 + T, T, T, N, K, gated, True, True)
        check(c, run(ctx, c, "gelu"), "gelu")
