"""dcut_rope_append against its formula in 64 bits.

Tolerance: one rounding to bf16 (half a step, 2^-8 relative) of a value whose fp32 computation is off by a few 2^-24 of
the rotated pair's length: angle 2^-23, cos/sin, two products and a sum, and the norm's sum of 128 squares: below 2^-18
of the pair's length in all.  So |err| <= 2^-8 |y| + 2^-17 |(a, b)|."""
import numpy as np
import pytest
import torch

from tests.plain_reference import bf16_values, prefix_len_of, rope_rows

pytestmark = pytest.mark.gpu


def _ctx(B, hq, hkv, d, pages=4096):
    from paper_2607_14647_b200 import binding
    return binding.Context(max_B=B, max_gamma=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_pages_per_req=pages)


def _i32(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _case(seed, counts, starts, hq, hkv, d, R, cap=None, layout="fused", norm=False, plens=None, cu_group=None, stride=None):
    """Inputs of one call; every touched page distinct, the rest of the table pointing anywhere in the pool."""
    rng = np.random.default_rng(seed)
    counts, starts = np.asarray(counts), np.asarray(starts)
    B, T = len(counts), int(counts.sum())
    cap = T if cap is None else cap
    req = np.repeat(np.arange(B), counts)
    cu = np.concatenate([[0], np.cumsum(counts)])
    pos = starts[req] + np.arange(T) - cu[req]
    pre = np.zeros(B, int) if plens is None else np.array([prefix_len_of(i, cu_group, plens) for i in range(B)])
    slot = pos - pre[req]
    touched = np.unique(req.astype(np.int64) * (1 << 32) + slot // 16)
    pool = len(touched) + 5
    table = rng.integers(0, pool, (B, (int(slot.max()) // 16 + 1) if stride is None else stride))
    table[touched >> 32, touched & 0xffffffff] = rng.permutation(pool)[: len(touched)]
    g = torch.Generator("cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    if layout == "fused":
        x = n(cap, hq + 2 * hkv, d)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    elif layout == "heads_first":
        q, k, v = n(hq, cap, d).transpose(0, 1), n(hkv, cap, d).transpose(0, 1), n(hkv, cap, d).transpose(0, 1)
    elif layout == "broadcast":
        q, k, v = n(cap, 1, d).expand(cap, hq, d), n(cap, 1, d).expand(cap, hkv, d), n(cap, hkv, d)
    else:
        q, k, v = n(cap, hq, d), n(cap, hkv, d), n(cap, hkv, d)
    freq = np.array([1.0e6 ** (-2.0 * e / max(R, 1)) for e in range(R // 2)])
    return dict(T=T, cap=cap, cu=cu, req=np.concatenate([req, np.full(cap - T, -1)]), pos=np.concatenate([pos, np.full(cap - T, -1)]),
                slot=slot, table=table, q=q, k=k, v=v, freq=freq, hq=hq, hkv=hkv, d=d, B=B,
                q_gain=1 + 0.2 * n(d) if norm else None, k_gain=1 + 0.2 * n(d) if norm else None,
                kc=n(pool, hkv, 16, d), vc=n(pool, hkv, 16, d), plens=plens, cu_group=cu_group)


def _call(ctx, c, interleaved=False, q_out=None, use_cu=True):
    from paper_2607_14647_b200 import binding
    groups = None
    if c["plens"] is not None:
        groups = binding.PrefixGroups(_i32(c["cu_group"]), _i32(c["plens"]), _i32(np.zeros((len(c["plens"]), 1))))
    freq = torch.tensor(c["freq"], dtype=torch.float64, device="cuda") if len(c["freq"]) else None
    c["keep"] = (freq, groups, _i32(c["table"]), _i32(c["req"]), _i32(c["pos"]), _i32(c["cu"]))
    return ctx.rope_append(c["q"], c["k"], c["v"], freq, c["kc"], c["vc"], c["keep"][2], c["keep"][3], c["keep"][4], c["cap"],
                           cu_q=c["keep"][5] if use_cu else None, interleaved=interleaved, q_gain=c["q_gain"], k_gain=c["k_gain"],
                           rms_eps=1e-6, groups=groups, q_out=q_out)


def _near(got, want, x):
    """x: the values before the rotation; a rotation does not change a head's length, which bounds the pair's."""
    pair = np.sqrt((x * x).sum(-1, keepdims=True)) if x is not None else 0
    lim = 2.0 ** -8 * np.abs(want) + 2.0 ** -17 * pair
    return (np.abs(got - want) <= lim).all()


def _check(c, q_out, kc0, vc0, interleaved=False):
    T, page = c["T"], c["table"][c["req"][: c["T"]], c["slot"] // 16]
    at = c["slot"] % 16
    gains = [None if g is None else bf16_values(g) for g in (c["q_gain"], c["k_gain"])]
    want_q = rope_rows(bf16_values(c["q"])[:T], c["pos"][:T], c["freq"], interleaved, gains[0], 1e-6)
    want_k = rope_rows(bf16_values(c["k"])[:T], c["pos"][:T], c["freq"], interleaved, gains[1], 1e-6)
    if q_out is not None:
        assert _near(bf16_values(q_out)[:T], want_q, want_q)
    kc, vc = bf16_values(c["kc"]), bf16_values(c["vc"])
    assert _near(kc[page, :, at], want_k, want_k)
    assert np.array_equal(vc[page, :, at], bf16_values(c["v"])[:T])
    # nothing else in the cache moved
    kc[page, :, at], vc[page, :, at] = 0, 0
    k0, v0 = kc0.copy(), vc0.copy()
    k0[page, :, at], v0[page, :, at] = 0, 0
    assert np.array_equal(kc, k0) and np.array_equal(vc, v0)


def _both(ctx, c, **kw):
    k0, v0 = bf16_values(c["kc"]), bf16_values(c["vc"])
    out = _call(ctx, c, **kw)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == 0
    _check(c, out, k0, v0, kw.get("interleaved", False))
    return out


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [0, 16, 64, 128])
@pytest.mark.parametrize("layout", ["fused", "dense", "heads_first", "broadcast"])
def test_layouts_and_rotary_widths(layout, R, interleaved):
    ctx = _ctx(4, 8, 2, 128)
    _both(ctx, _case(1, [1, 5, 17, 2], [0, 15, 1000, 31], 8, 2, 128, R, layout=layout, norm=R == 64), interleaved=interleaved)


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (16, 16, 64), (64, 8, 128), (20, 4, 128), (6, 2, 64), (1, 1, 128)])
@pytest.mark.parametrize("norm", [False, True])
def test_head_layouts(hq, hkv, d, norm):
    ctx = _ctx(3, hq, hkv, d)
    _both(ctx, _case(2, [1, 3, 16], [7, 100, 16], hq, hkv, d, d, norm=norm))


def test_one_token_and_a_long_prompt():
    ctx = _ctx(2, 8, 2, 128)
    _both(ctx, _case(3, [1], [0], 8, 2, 128, 128))
    _both(ctx, _case(4, [2501, 1], [0, 77], 8, 2, 128, 64, norm=True), interleaved=True)


def test_far_positions_keep_their_angle():
    ctx = _ctx(3, 4, 1, 128, pages=1 << 24)
    _both(ctx, _case(5, [9, 4, 3], [131072 - 3, 1000003, 8000000], 4, 1, 128, 128))


def test_padding_rows_and_rows_behind_the_last_are_left_alone():
    ctx = _ctx(3, 8, 2, 128)
    c = _case(6, [2, 1, 4], [3, 4, 5], 8, 2, 128, 128, cap=20)
    c["req"][c["T"]:], c["pos"][c["T"]:] = 99, -5             # rows past cu_q[B] are not looked at
    out = torch.full((20, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    _both(ctx, c, q_out=out)
    assert bool((out[c["T"]:] == 7).all())
    c["req"][c["T"]:] = -1                                    # without cu_q they are padding
    out.fill_(7)
    _both(ctx, c, q_out=out, use_cu=False)
    assert bool((out[c["T"]:] == 7).all())


def test_shared_prefix_moves_the_slot_not_the_angle():
    ctx = _ctx(6, 8, 2, 128)
    c = _case(7, [1, 2, 3, 4, 5, 6], [100, 117, 40, 41, 9, 12], 8, 2, 128, 128, plens=[100, 33, 0, 5], cu_group=[0, 2, 4, 4, 6])
    _both(ctx, c)


def test_keys_and_values_only_and_in_place():
    ctx = _ctx(2, 8, 2, 128)
    c = _case(8, [3, 4], [0, 16], 8, 2, 128, 128, layout="dense")
    q = c["q"]
    c["q"] = None
    k0, v0 = bf16_values(c["kc"]), bf16_values(c["vc"])
    assert _call(ctx, c) is None
    c["q"] = torch.zeros_like(q)
    torch.cuda.synchronize()
    _check(c, None, k0, v0)
    c["q"] = q.clone()
    want = _call(ctx, c)
    c["q"] = q
    got = _call(ctx, c, q_out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want)


def test_nan_and_infinity_pass_where_nothing_turns():
    ctx = _ctx(1, 8, 2, 128)
    c = _case(9, [4], [0], 8, 2, 128, 64, layout="dense")
    c["v"][1, 0, 3], c["v"][2, 1, 7], c["k"][0, 0, 100], c["q"][3, 2, 127] = float("nan"), float("inf"), float("-inf"), float("nan")
    out = _call(ctx, c)
    page, at = c["table"][0, 0], c["slot"] % 16
    vc, kc = c["vc"][page].float(), c["kc"][page].float()
    assert torch.isnan(vc[0, at[1], 3]) and vc[1, at[2], 7] == float("inf") and kc[0, at[0], 100] == float("-inf")
    assert torch.isnan(out[3, 2, 127].float()) and int(torch.isnan(out.float()).sum()) == 1


@pytest.mark.parametrize("what,code", [("page", 2), ("page_low", 2), ("column", 8), ("request", 8), ("position", 8), ("before_prefix", 8)])
def test_bad_tokens_are_reported_and_leave_no_trace(what, code):
    ctx = _ctx(3, 8, 2, 128)
    c = _case(10, [2, 1, 2], [20, 40, 60], 8, 2, 128, 128, plens=[16] if what == "before_prefix" else None, cu_group=[0, 3] if what == "before_prefix" else None)
    bad = 2                                                    # the token of request 1
    if what == "page":
        c["table"][1, c["slot"][bad] // 16] = c["kc"].shape[0]
    elif what == "page_low":
        c["table"][1, c["slot"][bad] // 16] = -1
    elif what == "column":
        c["pos"][bad] = 16 * c["table"].shape[1] + (16 if what == "before_prefix" else 0)
    elif what == "request":
        c["req"][bad] = 3
    elif what == "position":
        c["pos"][bad] = -1
    else:
        c["pos"][bad] = 15
    k0, v0 = bf16_values(c["kc"]), bf16_values(c["vc"])
    out = torch.full((5, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    _call(ctx, c, q_out=out)
    assert ctx.poll_device_status() == code and ctx.poll_device_status() == 0
    assert bool((out[bad] == 7).all())
    # the other tokens are in place, everything else untouched
    keep = np.array([0, 1, 3, 4])
    c2 = dict(c, T=4, q=c["q"][keep], k=c["k"][keep], v=c["v"][keep], req=c["req"][keep], pos=c["pos"][keep], slot=c["slot"][keep])
    _check(c2, out[keep], k0, v0)


def test_captured_and_replayed_on_another_stream():
    ctx = _ctx(3, 8, 2, 128)
    c = _case(11, [2, 1, 9], [20, 40, 60], 8, 2, 128, 128, norm=True)
    kc0, vc0 = c["kc"].clone(), c["vc"].clone()
    want = _call(ctx, c)
    kc1, vc1 = c["kc"].clone(), c["vc"].clone()
    c["kc"].copy_(kc0), c["vc"].copy_(vc0)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        ctx.rope_append(c["q"], c["k"], c["v"], c["keep"][0], c["kc"], c["vc"], c["keep"][2], c["keep"][3], c["keep"][4], c["cap"],
                        cu_q=c["keep"][5], q_gain=c["q_gain"], k_gain=c["k_gain"], q_out=out)
    assert not out.any()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(c["kc"], kc1) and torch.equal(c["vc"], vc1)


def test_pages_and_tokens_behind_two_to_the_31_elements():
    """The last pages of a cache of more than 2^31 elements, from q, k, v whose tokens lie far apart."""
    ctx = _ctx(4, 8, 8, 128)
    c = _case(77, [1, 5, 3, 2], [0, 15, 100, 31], 8, 8, 128, 128, layout="dense")
    want = _call(ctx, c)
    k_want, v_want = c["kc"].clone(), c["vc"].clone()
    pool, shift = c["kc"].shape[0], 2 ** 31 // (8 * 16 * 128) + 5
    c["table"] = c["table"] + shift
    for n in ("kc", "vc"):
        big = torch.empty((shift + pool, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
        big[shift:] = c[n]
        c[n] = big
    for n in ("q", "k", "v"):
        far = torch.empty((c["cap"], 1 << 28), dtype=torch.bfloat16, device="cuda")[:, : 8 * 128].view(c["cap"], 8, 128)
        far.copy_(c[n])
        c[n] = far
    c["kc"][shift:], c["vc"][shift:] = 0, 0
    got = _call(ctx, c)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == 0 and torch.equal(got, want)
    req, slot = c["req"][: c["T"]], c["slot"]
    page, at = c["table"][req, slot // 16], slot % 16
    assert torch.equal(c["kc"][page, :, at], k_want[page - shift, :, at]) and torch.equal(c["vc"][page, :, at], v_want[page - shift, :, at])


@pytest.mark.parametrize("cu_group,plens,bad_requests", [([0, 2], [32], [2]), ([1, 3], [32], [0]), ([0, 2, 1, 3], [16, 0, 16], [1]), ([0, 1, 3], [16, -16], [1, 2]),
                                                         ([0, 3, 3], [16, -16], [])])
def test_requests_that_not_exactly_one_group_covers_are_reported(cu_group, plens, bad_requests):
    """No group, two of them (borders out of order), a negative prefix length (of an empty group: nothing to report)."""
    ctx = _ctx(3, 8, 2, 128)
    c = _case(12, [2, 1, 2], [40, 50, 60], 8, 2, 128, 128, stride=8)
    rows = [r for r in range(5) if c["req"][r] not in bad_requests]
    slot = c["slot"] - np.array([next((p for p, lo, hi in zip(plens, cu_group, cu_group[1:]) if lo <= q < hi), 0) for q in c["req"]])
    c["table"] = np.arange(24).reshape(3, 8)
    g = torch.Generator("cuda").manual_seed(1)
    for n in ("kc", "vc"):
        c[n] = torch.randn((24, 2, 16, 128), generator=g, device="cuda").to(torch.bfloat16)
    c["plens"], c["cu_group"] = plens, cu_group
    k0, v0 = bf16_values(c["kc"]), bf16_values(c["vc"])
    out = torch.full((5, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    _call(ctx, c, q_out=out)
    assert ctx.poll_device_status() == (8 if bad_requests else 0)
    assert all(bool((out[r] == 7).all()) for r in range(5) if r not in rows)
    _check(dict(c, T=len(rows), q=c["q"][rows], k=c["k"][rows], v=c["v"][rows], req=c["req"][rows], pos=c["pos"][rows], slot=slot[rows]), out[rows], k0, v0)


def test_rows_past_the_capacity_are_reported():
    ctx = _ctx(3, 8, 2, 128)
    c = _case(13, [2, 1, 2], [40, 50, 60], 8, 2, 128, 128)
    c["cu"][-1] = 6
    k0, v0 = bf16_values(c["kc"]), bf16_values(c["vc"])
    out = _call(ctx, c)
    assert ctx.poll_device_status() == 10 and ctx.poll_device_status() == 0
    _check(c, out, k0, v0)


def test_one_token_from_a_row_of_any_length():
    """The first row of a buffer whose rows are no multiple of 8 elements apart."""
    ctx = _ctx(1, 8, 2, 128)
    c = _case(14, [1], [37], 8, 2, 128, 128, layout="dense")
    for n, h in (("q", 8), ("k", 2), ("v", 2)):
        rows = torch.zeros((2, h * 128 + 3), dtype=torch.bfloat16, device="cuda")
        rows[:1, : h * 128] = c[n].reshape(1, -1)
        c[n] = rows[:, : h * 128].view(2, h, 128)[:1]
        assert c[n].stride(0) % 8
    _both(ctx, c)
