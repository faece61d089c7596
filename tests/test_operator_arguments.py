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
