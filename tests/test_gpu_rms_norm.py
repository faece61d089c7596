"""dcut_rms_norm against its formula in 64 bits.

Tolerance.  u = 2^-24, the rounding of an fp32 operation.  h = x + residual: one rounding, u |h|.  The sum of squares adds n
positive terms, each relative error at most (n + 2 + 2) u whatever the order (a term's square carries h's error twice), and half
of that reaches 1 / sqrt; the quotient, the addition of eps, the root and the division add a rounding each: r is off by e_r =
((n + 4) / 2 + 4) u.  y = h gain r: three roundings and h's more, and one for 1 + gain: e_y = e_r + 5 u (with the gain's sum, where
1 + gain may cancel, exact in fp32: gain is bf16 of magnitude below 2^7 and above 2^-9 in these tests).  bf16 adds half a step, 2^-8 |y|.
scale: that of max |y|, and one rounding: e_y + u; without a norm u.
out8, times the row's own scale: y / scale has a rounding for each of 448 / max, the product, and the scale's own, 3 u of the value; the
rounding to e4m3 is half a step: 2^-4 of the value, or 2^-10 (half the smallest step 2^-9) below the normal range.
"""
import numpy as np
import pytest
import torch

from tests.plain_reference import bf16_values, rms_norm as plain

pytestmark = pytest.mark.gpu
NAN, U = float("nan"), 2.0 ** -24
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def context():
    from paper_2607_14647_b200 import binding
    return binding.Context(max_B=8, max_gamma=4)


def view(g, rows, cols, pad, scale=1.0, shift=0):
    """A view of rows `cols + pad` apart, `shift` elements into its buffer; NaN beside the rows."""
    buf = torch.full((rows * (cols + pad) + shift,), NAN, dtype=BF16, device="cuda")
    v = buf[shift:].view(rows, cols + pad)[:, :cols]
    v.copy_(scale * torch.randn((rows, cols), generator=g, device="cuda"))
    return v


def run(ctx, x, T, cap, normed=True, gain=None, residual=None, outs="hb8", pad=0, eps=1e-6, plus_one=False, cu="some"):
    """Every output in a buffer of sevens (rows `pad` apart), and the buffers."""
    w = x.shape[1]
    buf = dict(h=torch.full((cap + 1, w + pad), 7.0, dtype=BF16, device="cuda"), b=torch.full((cap + 1, w + pad), 7.0, dtype=BF16, device="cuda"))
    buf["8"] = torch.full((cap + 1, w + pad), 7.0, device="cuda").to(F8)
    buf["s"] = torch.full((cap + 1,), 7.0, device="cuda")
    o = {k: buf[k][:, :w] if k in outs else None for k in "hb8"}
    cu_q = None if cu is None else torch.tensor([0, T // 2, T], dtype=torch.int32, device="cuda")
    kw = dict(residual=residual, h_out=o["h"], out=o["b"], out8=o["8"], scale8=buf["s"] if "8" in outs else None)
    if normed:
        ctx.rms_norm(x, cu_q, cap, gain=gain, rms_eps=eps, gain_plus_one=plus_one, **kw)
    elif "8" in outs:
        ctx.quantize(x, cu_q, cap, **kw)
    assert ctx.poll_device_status() == 0
    return o, buf


def check(o, buf, x, T, normed=True, gain=None, residual=None, eps=1e-6, plus_one=False):
    n = x.shape[1]
    h, y = plain(bf16_values(x[:T]), None if residual is None else bf16_values(residual[:T]), normed, None if gain is None else bf16_values(gain), eps, plus_one)
    e = (((n + 4) / 2 + 4) + 5) * U if normed else U

    def near(got, want, tol):
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()

    if o["h"] is not None:
        near(bf16_values(o["h"])[:T], h, (1 + 2.0 ** -8) * U * np.abs(h) + 2.0 ** -8 * np.abs(h) + 1e-40)
    if o["b"] is not None:
        near(bf16_values(o["b"])[:T], y, (1 + 2.0 ** -8) * e * np.abs(y) + 2.0 ** -8 * np.abs(y) + 1e-40)
    if o["8"] is not None:
        s = buf["s"].cpu().numpy().astype(np.float64)[:T]
        want = np.maximum(np.abs(y).max(1), 2.0 ** -100) / 448
        near(s, want, (e + 2 * U) * want)
        q = o["8"][:T].float().cpu().numpy().astype(np.float64)
        z = y / s[:, None]                                             # in units of the row's own scale
        near(q, z, np.maximum(2.0 ** -4 * np.abs(z), 2.0 ** -10) + 1.1 * (e + 3 * U) * np.abs(z))
    for name, t in buf.items():                                         # rows behind the last token and beside the row
        wrote = o["8" if name == "s" else name] is not None
        rest = t if not wrote else t[T:]
        assert (rest.float() == 7).all()
        if wrote and t.dim() == 2:
            assert (t[:, n:].float() == 7).all()


WIDTHS = [1, 7, 8, 31, 64, 65, 255, 256, 264, 1000, 2047, 2048, 2051, 4096, 4104, 8200, 12288, 16385, 32768]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("normed,residual", [(True, True), (True, False), (False, False)])
def test_widths(width, normed, residual):
    g = torch.Generator("cuda").manual_seed(width)
    T, cap, pad = 5, 7, -width % 8
    x, r = view(g, cap, width, pad, 3.0), view(g, cap, width, pad) if residual else None
    gain = 1 + 0.2 * torch.randn(width, generator=g, device="cuda").to(BF16) if normed else None
    ctx = context()
    for out_pad in (0, pad + 8 if pad else 16):
        o, buf = run(ctx, x, T, cap, normed, gain, r, pad=out_pad)
        check(o, buf, x, T, normed, gain, r)


@pytest.mark.parametrize("T,cap", [(0, 3), (1, 1), (2, 9), (129, 200), (1000, 1000), (4097, 4100)])
def test_row_counts(T, cap):
    g = torch.Generator("cuda").manual_seed(T)
    for width in (96, 1024):
        x, r = view(g, cap, width, 0), view(g, cap, width, 0)
        o, buf = run(context(), x, T, cap, residual=r)
        check(o, buf, x, T, residual=r)


@pytest.mark.parametrize("outs", ["h", "b", "8", "hb", "h8", "b8"])
@pytest.mark.parametrize("normed", [True, False])
def test_each_output_alone(outs, normed):
    g = torch.Generator("cuda").manual_seed(3)
    x, r = view(g, 6, 520, 0), view(g, 6, 520, 0)
    if not normed and "8" not in outs:
        return
    o, buf = run(context(), x, 4, 6, normed, residual=r, outs=outs)
    check(o, buf, x, 4, normed, residual=r)


@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 0), (8, 3), (24, 8), (5, 1)])
def test_strides_and_odd_places(pad, shift):
    g = torch.Generator("cuda").manual_seed(pad)
    x, r = view(g, 5, 200, pad, shift=shift), view(g, 5, 200, 0)
    gain = torch.randn(200 + 3, generator=g, device="cuda").to(BF16)[3:]
    for plus_one in (False, True):
        o, buf = run(context(), x, 5, 5, gain=gain, residual=r, plus_one=plus_one, pad=pad)
        check(o, buf, x, 5, gain=gain, residual=r, plus_one=plus_one)


def test_all_rows_without_cu_q():
    g = torch.Generator("cuda").manual_seed(4)
    x = view(g, 9, 300, 4)
    o, buf = run(context(), x, 9, 9, False, cu=None)
    check(o, buf, x, 9, False)


@pytest.mark.parametrize("width", [328, 331, 4096])
def test_in_place_over_x_and_the_residual(width):
    ctx, T = context(), 6
    for over in ("residual", "x"):
        g = torch.Generator("cuda").manual_seed(5)
        x, r = view(g, T, width, 8), view(g, T, width, 8)
        x0, r0 = x.clone(), r.clone()
        cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        out = x if over == "residual" else torch.empty_like(x0)
        h = r if over == "residual" else x
        ctx.rms_norm(x, cu, T, residual=r, h_out=h, out=out)
        hw, y = plain(bf16_values(x0), bf16_values(r0), True, None, 1e-6, False)
        assert (np.abs(bf16_values(h) - hw) <= 2.0 ** -8 * 1.01 * np.abs(hw)).all()
        assert (np.abs(bf16_values(out) - y) <= (2.0 ** -8 + (width / 2 + 11) * U) * 1.01 * np.abs(y)).all()


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e15, 1e19, 1e30, 3e37])
def test_sizes_of_values(scale):
    """Squares that vanish beside eps, squares that overflow."""
    g = torch.Generator("cuda").manual_seed(6)
    for width in (77, 256, 5000):
        x = view(g, 4, width, -width % 8, scale)
        o, buf = run(context(), x, 4, 4, outs="hb8")
        check(o, buf, x, 4)
        o, buf = run(context(), x, 4, 4, False, outs="hb8")
        check(o, buf, x, 4, False)


def test_rows_of_zeros_and_of_one_value():
    x = torch.zeros((4, 264), dtype=BF16, device="cuda")
    x[1, 263] = -3.0
    x[2] = 0.5
    for normed in (True, False):
        o, buf = run(context(), x, 4, 4, normed)
        check(o, buf, x, 4, normed)
        assert (o["8"][0].float() == 0).all() and o["8"][1, 263].float() == -448


def test_infinities_and_nan_stay_in_their_rows():
    g = torch.Generator("cuda").manual_seed(7)
    for width in (40, 1000, 4096):
        x = view(g, 6, width, 0)
        clean = x.clone()
        x[1, width - 1], x[2, 3], x[4, 0] = NAN, float("inf"), -float("inf")
        ctx = context()
        for normed in (True, False):
            o, buf = run(ctx, x, 6, 6, normed)
            ref, rbuf = run(ctx, clean, 6, 6, normed)
            for r in range(6):
                if r in (0, 3, 5):
                    assert torch.equal(o["b"][r], ref["b"][r]) and torch.equal(o["8"][r].view(torch.uint8), ref["8"][r].view(torch.uint8))
                    assert buf["s"][r] == rbuf["s"][r]
                    continue
                assert torch.isnan(buf["s"][r]) and torch.isnan(o["8"][r].float()).all()
                bad = torch.isnan(x[r].float()) if not normed else (~torch.isfinite(x[r].float()) if r != 1 else torch.ones(width, dtype=torch.bool, device="cuda"))
                got = o["b"][r].float()
                assert torch.equal(torch.isnan(got), bad)
                if normed and r != 1:
                    assert (got[~bad] == 0).all()                      # x / infinity


def test_a_packing_above_the_cap_is_reported():
    ctx = context()
    x = torch.ones((5, 64), dtype=BF16, device="cuda")
    out = torch.full((5, 64), 7.0, dtype=BF16, device="cuda")
    ctx.rms_norm(x, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), 3, out=out)
    assert ctx.poll_device_status() == 10
    assert (out[:3] == 1).all() and (out[3:] == 7).all()


def test_rows_behind_2_31_elements():
    ctx, width, T = context(), 32768, 65540
    x = torch.zeros((T, width), dtype=BF16, device="cuda")
    g = torch.Generator("cuda").manual_seed(8)
    x[-3:] = torch.randn((3, width), generator=g, device="cuda").to(BF16)
    out8, scale8 = ctx.quantize(x, None, T)
    o, s = out8[-3:], scale8[-3:]
    check({"h": None, "b": None, "8": o}, {"s": s}, x[-3:], 3, False)


def test_another_stream_and_a_captured_call():
    g = torch.Generator("cuda").manual_seed(9)
    ctx, x, r = context(), view(g, 30, 512, 0), view(g, 30, 512, 0)
    eager, _ = run(ctx, x, 21, 30, residual=r)
    cu = torch.tensor([0, 21], dtype=torch.int32, device="cuda")
    out, out8, s = torch.zeros((30, 512), dtype=BF16, device="cuda"), torch.zeros((30, 512), device="cuda").to(F8), torch.zeros(30, device="cuda")
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        ctx.rms_norm(x, cu, 30, residual=r, out=out, out8=out8, scale8=s)
    for T in (21, 5):
        cu[1] = T
        out.zero_()
        graph.replay()
        assert torch.equal(out[:T], eager["b"][:T]) and (out[T:] == 0).all()
        assert torch.equal(out8[:T].view(torch.uint8), eager["8"][:T].view(torch.uint8))


@pytest.mark.parametrize("scale,gain_scale", [(100.0, 5e36), (1e10, 1e36), (1e-3, 5e36), (1e37, 1e20), (1e37, 1e30)])
def test_gains_whose_product_with_h_overflows_where_y_does_not(scale, gain_scale):
    """h gain is above fp32's largest value, its squares' sum is not (or is too): y is an ordinary number of bf16."""
    g = torch.Generator("cuda").manual_seed(12)
    for width in (77, 256, 5000, 20000):
        x, gain = view(g, 4, width, -width % 8, scale), (gain_scale * torch.randn(width, generator=g, device="cuda")).to(BF16)
        o, buf = run(context(), x, 4, 4, gain=gain)
        check(o, buf, x, 4, gain=gain)
