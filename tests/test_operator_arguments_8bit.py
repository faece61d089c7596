"""Arguments that the binding of the 8-bit and adapter operators checks itself, and what it passes on (no GPU)."""
import pytest
import torch

from paper_2607_14647_b200 import binding as b
from tests.test_operator_arguments import B, BF16, I32, T, ctx  # noqa: F401  (ctx is a fixture)


@pytest.fixture
def ctx8(ctx, monkeypatch):  # noqa: F811
    for name in ("dcut_rms_norm", "dcut_linear8", "dcut_lora"):
        monkeypatch.setattr(b._lib, name, lambda *a: ctx.calls.append(a) or b.OK)
    return ctx


def z(*shape, dtype=BF16):
    return torch.zeros(shape, dtype=dtype)


F32 = torch.float32
CU = torch.zeros(B + 1, dtype=I32)
NORM = dict(x=z(T, 40), cu_q=CU, T_cap=T, gain=z(40), out8=b.rows8(T, 40, "cpu"), scale8=z(T, dtype=F32))
LINEAR8 = dict(a=b.rows8(T, 40, "cpu"), a_scale=z(T, dtype=F32), w=b.rows8(24, 40, "cpu"), w_scale=z(24, dtype=F32), cu_q=CU, T_cap=T)
LORA = dict(x=z(T, 40), a=z(2, 16, 40), b=z(2, 24, 8), adapter=z(B, dtype=I32), base=z(T, 24), cu_q=CU, T_cap=T, slices=[10, 24])


def test_good_arguments_pass(ctx8):
    ctx8.rms_norm(**NORM)
    ctx8.linear8(**LINEAR8)
    ctx8.lora(**LORA)
    n, l, a = (t.from_buffer_copy(c[1]) for t, c in zip((b.NormArgs, b.Linear8Args, b.LoraArgs), ctx8.calls))
    assert (n.width, n.ldx, n.ld8, n.normed, n.gain_plus_one) == (40, 40, 48, 1, 0)
    assert (l.N, l.K, l.lda, l.ldw, l.ldo) == (24, 40, 48, 48, 24)
    assert (a.n_adapters, a.rank, a.n_slices, list(a.slice_end)[:2], a.K, a.lda, a.ldbase) == (2, 8, 2, [10, 24], 40, 40, 24)
    assert [c[3] for c in ctx8.calls] == [B, B, B] and [c[4] for c in ctx8.calls] == [T, T, T]


@pytest.mark.parametrize("wrong", [
    dict(x=z(T - 1, 40)), dict(x=z(T, 40, dtype=torch.float16)), dict(gain=z(41)), dict(residual=z(T, 39)), dict(out=z(T - 1, 40)), dict(h_out=z(T, 41)),
    dict(out8=z(T, 40)), dict(scale8=z(T - 1, dtype=F32)), dict(scale8=z(T)), dict(cu_q=z(B + 1)), dict(x=z(40, T).t())])
def test_rms_norm_refuses(ctx8, wrong):
    with pytest.raises(AssertionError):
        ctx8.rms_norm(**dict(NORM, **wrong))
    assert not ctx8.calls


@pytest.mark.parametrize("wrong", [
    dict(a=z(T, 40)), dict(a=b.rows8(T - 1, 40, "cpu")), dict(a=b.rows8(T, 41, "cpu")), dict(a_scale=z(T - 1, dtype=F32)), dict(w_scale=z(25, dtype=F32)),
    dict(bias=z(23)), dict(bias2=z(25)), dict(residual=z(T, 23)), dict(out=z(T, 25)), dict(w2=b.rows8(23, 40, "cpu"), w2_scale=z(23, dtype=F32)),
    dict(w2=b.rows8(24, 40, "cpu"), w2_scale=z(23, dtype=F32)), dict(w2=b.rows8(24, 64, "cpu")[:, :40], w2_scale=z(24, dtype=F32))])
def test_linear8_refuses(ctx8, wrong):
    with pytest.raises(AssertionError):
        ctx8.linear8(**dict(LINEAR8, **wrong))
    assert not ctx8.calls


@pytest.mark.parametrize("wrong", [
    dict(x=z(T, 41)), dict(a=z(2, 8, 40)), dict(a=z(3, 16, 40)), dict(a=z(16, 2, 40).transpose(0, 1)), dict(b=z(2, 23, 8)), dict(b=z(2, 24, 16)),
    dict(adapter=z(B - 1, dtype=I32)), dict(adapter=z(B)), dict(base=z(T, 23)), dict(base=z(T - 1, 24)), dict(scale=z(3, dtype=F32)), dict(slices=[10, 23]),
    dict(slices=[4, 8, 12, 16, 24]), dict(out=z(T, 12)), dict(gated=True, out=z(T, 24))])
def test_lora_refuses(ctx8, wrong):
    with pytest.raises(AssertionError):
        ctx8.lora(**dict(LORA, **wrong))
    assert not ctx8.calls


def test_rows_of_single_rows_and_padded_views(ctx8):
    ctx8.rms_norm(z(2, 43)[:, :40][:1], CU, 1, out=z(1, 40))
    assert b.NormArgs.from_buffer_copy(ctx8.calls[-1][1]).ldx == 40
    ctx8.lora(**dict(LORA, x=z(T, 56)[:, :40], a=z(2, 16, 48)[:, :, :40], base=z(T, 31)[:, :24], out=z(T, 27)[:, :24]))
    a = b.LoraArgs.from_buffer_copy(ctx8.calls[-1][1])
    assert (a.ldx, a.lda, a.ldbase, a.ldo) == (56, 48, 31, 27)
