"""Arguments that the binding of the attention-block operators checks itself, and what it passes on (no GPU: the library's
entry points are replaced by recorders)."""
import ctypes as C

import pytest
import torch

from paper_2607_14647_b200 import binding as b

HQ, HKV, D, B, T = 8, 2, 64, 3, 5
BF16, I32 = torch.bfloat16, torch.int32


@pytest.fixture
def ctx(monkeypatch):
    """A context whose tensors live on the CPU and whose calls are recorded instead of made."""
    c = object.__new__(b.Context)
    c.device, c._shape, c._h, c.limits = -1, (HQ, HKV, D), None, b.Limits(B, 4, HQ, HKV, D, 16, 8, 0, 0, 0)
    c._stream = lambda: 0
    c.calls = []
    for name in ("dcut_rope_append", "dcut_prefix_attn", "dcut_linear"):
        monkeypatch.setattr(b._lib, name, lambda *a: c.calls.append(a) or b.OK)
    return c


def caches(shape=(6, HKV, 16, D)):
    return torch.zeros(shape, dtype=BF16), torch.zeros(shape, dtype=BF16)


def groups():
    return b.PrefixGroups.__new__(b.PrefixGroups)


def prefix_groups():
    g = groups()
    g.device, g.rec = -1, b.PrefixGroupsRec(1, 1, 1, 1, 1)
    return g


def append(ctx, kc, vc, q=None, k=None, v=None, T_cap=T, **kw):
    n = lambda h: torch.zeros((T, h, D), dtype=BF16)
    i = lambda *s: torch.zeros(s, dtype=I32)
    return ctx.rope_append(n(HQ) if q is None else q, n(HKV) if k is None else k, n(HKV) if v is None else v, None, kc, vc, i(B, 8), i(T), i(T), T_cap,
                           **kw)


def attn(ctx, kc, vc, **kw):
    i = lambda *s: torch.zeros(s, dtype=I32)
    return ctx.prefix_attn(torch.zeros((T, HQ, D), dtype=BF16), kc, vc, i(B, 8), i(B), i(B + 1), T, prefix_groups(), **kw)


WRONG = [(6, HKV, D, 16), (6, 16, HKV, D), (6, HKV, 8, D), (6, HKV + 1, 16, D), (6, 1, 16, D), (6, HKV, 16, D // 2), (6, HKV, 16 * D), (6, 1, HKV, 16, D)]


@pytest.mark.parametrize("call", [append, attn])
@pytest.mark.parametrize("shape", WRONG)
def test_caches_of_another_layout_are_refused(ctx, call, shape):
    with pytest.raises(AssertionError, match="caches must be"):
        call(ctx, *caches(shape))
    assert not ctx.calls


@pytest.mark.parametrize("call", [append, attn])
def test_caches_of_two_sizes_are_refused_and_the_context_s_own_layout_is_taken(ctx, call):
    with pytest.raises(AssertionError, match="caches must be"):
        call(ctx, caches()[0], caches((7, HKV, 16, D))[1])
    call(ctx, *caches())
    assert len(ctx.calls) == 1 and ctx.calls[0][6 if call is append else 4] == 6          # num_pages


def test_strides_of_a_single_token_or_head_say_nothing(ctx):
    """The first row of a buffer whose rows are no multiple of 8 apart; one key head with any stride."""
    q = torch.zeros((2, HQ * D + 3), dtype=BF16)[:, : HQ * D].view(2, HQ, D)[:1]
    assert q.stride(0) % 8
    append(ctx, *caches(), q=q, k=torch.zeros((1, HKV, D), dtype=BF16), v=torch.zeros((1, HKV, D), dtype=BF16), T_cap=1)
    x = ctx.calls[-1][1]._obj
    assert (x.q_token_stride, x.q_head_stride, x.k_token_stride, x.k_head_stride) == (0, D, 0, D)
    ctx._shape = (HQ, 1, D)
    one = torch.zeros((T, 2 * D), dtype=BF16).as_strided((T, 1, D), (2 * D, 5, 1))
    append(ctx, *caches((6, 1, 16, D)), k=one, v=torch.zeros((T, 1, D), dtype=BF16))
    x = ctx.calls[-1][1]._obj
    assert (x.q_token_stride, x.k_token_stride, x.k_head_stride, x.v_token_stride, x.v_head_stride) == (HQ * D, 2 * D, 0, D, 0)
