"""dcut_rms_norm's 8-bit rows, code by code: out8 = e4m3(y / scale8[r]) with the scale that the call stores.

No tolerance: without a norm y is one fp32 sum, or x itself; with one, rows of +-1 and rms_eps = 3 make the factor 1 / sqrt(1 + 3) = 1/2, so that
y = +-gain / 2 is exact.  The quotient is then one fp32 division and one rounding to e4m3, formed here on the CPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


def context():
    from paper_2607_14647_b200 import binding
    return binding.Context(max_B=8, max_gamma=4)


def expected(y):
    """(codes, scales) of fp32 rows."""
    y = y.cpu()
    scale = y.abs().amax(1).clamp(min=2.0 ** -100) / 448
    return (y / scale[:, None]).clamp(-448, 448).to(F8).view(torch.uint8), scale


def same(out8, scale8, y):
    codes, scale = expected(y)
    assert torch.equal(scale8.cpu(), scale)
    got = out8.contiguous().view(torch.uint8).cpu()
    assert torch.equal(got, codes), f"{int((got != codes).sum())} of {codes.numel()} codes differ"


@pytest.mark.parametrize("width,pad,shift", [(40, 0, 0), (256, 0, 0), (2051, 0, 0), (4096, 0, 0), (4096, 3, 1), (12288, 0, 0), (20000, 8, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_quantised_rows(width, pad, shift, residual):
    g = torch.Generator("cuda").manual_seed(width + pad)
    T = 64
    x = torch.empty(T * (width + pad) + shift, dtype=BF16, device="cuda")[shift:].view(T, width + pad)[:, :width]
    x.copy_(torch.randn((T, width), generator=g, device="cuda") * torch.exp(8 * torch.randn((T, 1), generator=g, device="cuda")))
    r = torch.randn((T, width), generator=g, device="cuda").to(BF16) if residual else None
    out8, scale8 = context().quantize(x, None, T, residual=r)
    same(out8, scale8, x.float() + r.float() if residual else x.float())


@pytest.mark.parametrize("scale", [1e-38, 2.0 ** -101, 1e-30, 1e30, 1e37])
def test_small_and_large_rows(scale):
    g = torch.Generator("cuda").manual_seed(3)
    x = (scale * torch.randn((32, 1000), generator=g, device="cuda")).to(BF16)
    out8, scale8 = context().quantize(x, None, 32)
    same(out8, scale8, x.float())


@pytest.mark.parametrize("width", [96, 4096, 12288])
def test_normed_rows(width):
    from paper_2607_14647_b200 import binding
    g = torch.Generator("cuda").manual_seed(width)
    T = 16
    x = (2.0 * torch.randint(0, 2, (T, width), generator=g, device="cuda") - 1).to(BF16)
    gain = (0.2 * torch.randn(width, generator=g, device="cuda") + 1).to(BF16)
    out8, scale8 = binding.rows8(T, width), torch.empty(T, device="cuda")
    context().rms_norm(x, None, T, gain=gain, rms_eps=3.0, out8=out8, scale8=scale8)
    same(out8, scale8, x.float() * gain.float() * 0.5)


def test_zeros_keep_their_sign():
    x = torch.tensor([0.0, -0.0, 1.0, -1.0] * 70, device="cuda").to(BF16).view(1, -1).expand(3, -1).contiguous()
    x[1] *= 2.0 ** -120
    x[2].mul_(0)                                                         # only zeros, of both signs
    out8, scale8 = context().quantize(x, None, 3)
    same(out8, scale8, x.float())


@pytest.mark.parametrize("seed", range(4))
def test_many_sums(seed):
    """33 million fp32 values of rows of all sizes, against fp32 division by the stored scales."""
    g = torch.Generator("cuda").manual_seed(seed)
    T, width = 4096, 8192
    size = 2.0 ** torch.randint(-90, 90, (T, 1), generator=g, device="cuda").float()
    x, r = ((size * torch.randn((T, width), generator=g, device="cuda") * f).to(BF16) for f in (1.0, 2.0 ** -seed))
    out8, scale8 = context().quantize(x, None, T, residual=r)
    y = x.float() + r.float()
    assert torch.equal(scale8.cpu(), y.abs().amax(1).cpu() / 448)
    want = (y / scale8[:, None]).clamp(-448, 448).to(F8).view(torch.uint8)
    assert torch.equal(out8.contiguous().view(torch.uint8), want)
