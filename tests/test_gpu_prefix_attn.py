"""dcut_prefix_attn against its formula in 64 bits.

Tolerance.  The output is rounded to bf16 once: half a step, 2^-8 |y|.  Each softmax weight is rounded to bf16 once before
it meets V: at most 2^-8 of the weighted mean A of |v|.  A score is an fp32 sum of D exact products: off by at most
E = D 2^-23 scale sum_c |q_c k_c|, which moves a weight by a factor e^E and the output by 2 E A.  Exponentials, sums and the
merges of parts: a few 2^-22 each, below 2^-15 A in all.  The log-sum-exp sees E, 2^-18 of those, and 2^-21 of its value.
"""
import numpy as np
import pytest
import torch

from tests.plain_reference import bf16_values, prefix_attn as plain

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _i32(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def make_case(seed, counts, own, sizes, plens, hq, hkv, d, cap=None, q_scale=1.0, poison=True, extra_pages=3):
    """counts: rows per request; own: own context per request; sizes / plens: requests and prefix length per group."""
    rng = np.random.default_rng(seed)
    counts, own, sizes, plens = (np.asarray(x) for x in (counts, own, sizes, plens))
    B, T, G = len(counts), int(counts.sum()), len(sizes)
    group = np.repeat(np.arange(G), sizes)
    cu_group = np.concatenate([[0], np.cumsum(sizes)])
    pages = -(-(own + counts) // 16)
    shared = -(-plens // 16)
    pool = int(pages.sum() + shared.sum()) + extra_pages
    free = rng.permutation(pool)
    # (columns behind a request's pages hold numbers that are no pages: they must not be looked at)
    table, ptable = np.full((B, int(pages.max()) + 1), 1 << 30), np.full((G, int(shared.max()) + 1), -7)
    at = 0
    for rows, need in ((table, pages), (ptable, shared)):
        for i, n in enumerate(need):
            rows[i, :n] = free[at:at + n]
            at += n
    g = torch.Generator("cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    c = dict(T=T, cap=T if cap is None else cap, counts=counts, hq=hq, hkv=hkv, d=d, B=B, G=G, table=table, ptable=ptable, cu_group=cu_group,
             plens=plens, ctx=plens[group] + own, cu=np.concatenate([[0], np.cumsum(counts)]), kc=n(pool, hkv, 16, d), vc=n(pool, hkv, 16, d))
    c["q"] = (q_scale * n(c["cap"], hq, d)).to(torch.bfloat16)
    c["kc_plain"], c["vc_plain"] = bf16_values(c["kc"]), bf16_values(c["vc"])
    if poison:                                        # what lies behind a prefix's end, and in pages nobody owns
        for i, p in enumerate(plens):
            if p % 16:
                c["kc"][ptable[i, p // 16], :, p % 16:] = NAN
                c["vc"][ptable[i, p // 16], :, p % 16:] = NAN
        for j in free[at:]:
            c["kc"][int(j)], c["vc"][int(j)] = NAN, NAN
    return c


def make_ctx(c, max_gamma=None, groups=None):
    from paper_2607_14647_b200 import binding
    ctx = binding.Context(max_B=c["B"], max_gamma=max(1, int(c["counts"].max()) - 1) if max_gamma is None else max_gamma, n_q_heads=c["hq"],
                          n_kv_heads=c["hkv"], head_dim=c["d"], max_pages_per_req=max(c["table"].shape[1], c["ptable"].shape[1]))
    ctx.enable_prefix_attn(c["G"] if groups is None else groups)
    return ctx


def device_args(c):
    from paper_2607_14647_b200 import binding
    return dict(block_table=_i32(c["table"]), ctx_lens=_i32(c["ctx"]), cu_q=_i32(c["cu"]), T_cap=c["cap"],
                groups=binding.PrefixGroups(_i32(c["cu_group"]), _i32(c["plens"]), _i32(c["ptable"])))


def check(c, out, lse, scale=None, rows=None):
    d = c["d"]
    scale = d ** -0.5 if scale is None else scale
    want, want_lse, A, qk = plain(bf16_values(c["q"]), c["kc_plain"], c["vc_plain"], c["table"], c["ctx"], c["cu"], c["cu_group"], c["plens"], c["ptable"], scale)
    got = bf16_values(out)[: c["T"]]
    want, want_lse, A, qk = want[: c["T"]], want_lse[: c["T"]], A[: c["T"]], qk[: c["T"]]
    E = d * 2.0 ** -23 * qk
    lim = 2.0 ** -8 * (np.abs(want) + A) + (2 * E[..., None] + 2.0 ** -15) * A
    err = np.abs(got - want)
    assert (err <= lim).all(), f"worst err / limit {np.nanmax(err / lim)}, nan {np.isnan(got).sum()}"
    if lse is not None:
        l = lse.cpu().numpy().astype(np.float64)[: c["T"]]
        llim = E + 2.0 ** -18 + 2.0 ** -21 * np.abs(want_lse)
        assert (np.abs(l - want_lse) <= llim).all(), np.abs(l - want_lse).max()


def run(c, ctx=None, want_lse=True, **kw):
    ctx = ctx or make_ctx(c)
    out = torch.full((c["cap"], c["hq"], c["d"]), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c["cap"], c["hq"]), 7.0, device="cuda") if want_lse else None
    ctx.prefix_attn(c["q"], c["kc"], c["vc"], out=out, lse=lse, **device_args(c), **kw)
    torch.cuda.synchronize()
    assert ctx.poll_device_status() == 0
    assert bool((out[c["T"]:] == 7).all()) and (lse is None or bool((lse[c["T"]:] == 7).all()))
    return out, lse


@pytest.mark.parametrize("length", [1, 15, 16, 17, 127, 128, 129, 255, 300, 1000])
@pytest.mark.parametrize("d", [128, 64])
def test_one_group_every_length(length, d):
    c = make_case(1, [3, 1, 5], [0, 7, 40], [3], [length], 8, 2, d)
    check(c, *run(c))


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (64, 8, 128), (8, 8, 64), (16, 1, 128), (6, 2, 64), (20, 4, 128), (9, 1, 128), (1, 1, 64), (24, 8, 128)])
def test_head_layouts(hq, hkv, d):
    deep = min(17, 144 // (hq // hkv))
    rng = np.random.default_rng(hq)
    c = make_case(2, rng.integers(1, deep + 1, 13), rng.integers(0, 200, 13), [13], [333], hq, hkv, d)
    check(c, *run(c))


@pytest.mark.parametrize("sizes,plens", [([4, 3, 5], [200, 0, 77]), ([0, 6, 0, 6], [50, 130, 999, 16]), ([1] * 12, list(range(0, 240, 20))), ([12], [0])])
def test_groups(sizes, plens):
    rng = np.random.default_rng(3)
    c = make_case(3, rng.integers(1, 18, 12), rng.integers(0, 300, 12), sizes, plens, 8, 2, 128)
    check(c, *run(c))


@pytest.mark.parametrize("B", [1, 2, 31, 70])
def test_single_tokens(B):
    """One row per request: tiles that are nearly empty, exactly one, and the odd last one."""
    rng = np.random.default_rng(B)
    c = make_case(4, [1] * B, rng.integers(0, 100, B), [B], [700], 8, 2, 128)
    check(c, *run(c))


def test_no_own_context_at_all():
    c = make_case(5, [1, 4, 17], [0, 0, 0], [3], [160], 8, 2, 128)
    check(c, *run(c))


@pytest.mark.parametrize("tokens", [63, 64, 65, 129, 400])
def test_tiles_of_whole_and_cut_units(tokens):
    """32q / 4kv: 16 tokens a tile; odd and even numbers of tiles, long enough to be cut over many SMs."""
    deep = 17
    B = -(-tokens // deep)
    counts = np.full(B, deep)
    counts[-1] = tokens - deep * (B - 1)
    c = make_case(6, counts, np.arange(B) % 50, [B], [2500], 32, 4, 128)
    check(c, *run(c))


def test_large_scores_move_the_maximum():
    """Scores of +-100 and more: the running maximum moves and the accumulator is rescaled; late keys dominate."""
    c = make_case(7, [5, 9], [30, 0], [2], [1500], 8, 2, 128, q_scale=12.0)
    check(c, *run(c))
    c = make_case(8, [5, 9], [30, 0], [2], [1500], 8, 2, 128)
    ramp = torch.linspace(0.1, 4.0, 1500, device="cuda")
    for j in range(1500):
        c["kc"][int(c["ptable"][0, j // 16]), :, j % 16] = (c["q"][0, :2].float() * ramp[j]).to(torch.bfloat16)
    c["kc_plain"] = np.nan_to_num(bf16_values(c["kc"]))
    check(c, *run(c))


def test_scale_and_no_lse():
    c = make_case(9, [2, 3], [5, 6], [2], [90], 8, 2, 128)
    out, _ = run(c, want_lse=False, scale=0.3)
    check(c, out, None, scale=0.3)


def test_rows_behind_the_last_stay():
    c = make_case(10, [2, 3, 1], [5, 6, 70], [2, 1], [90, 33], 8, 2, 128, cap=17)
    check(c, *run(c, make_ctx(c, max_gamma=6)))


def test_equals_verify_attn_without_a_prefix():
    rng = np.random.default_rng(11)
    c = make_case(11, rng.integers(1, 18, 20), rng.integers(0, 800, 20), [20], [0], 32, 8, 128)
    ctx = make_ctx(c)
    out, lse = run(c, ctx)
    lse2 = torch.empty_like(lse)
    a = device_args(c)
    want = ctx.verify_attn(c["q"], c["kc"], c["vc"], a["block_table"], a["ctx_lens"], a["cu_q"], c["cap"], lse=lse2)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    np.testing.assert_allclose(lse.cpu().numpy(), lse2.cpu().numpy(), rtol=0, atol=2.0 ** -20)


def test_the_same_bits_every_time_and_between_other_calls():
    c = make_case(12, [17] * 20, np.arange(20) * 13, [20], [1999], 32, 8, 128)
    other = make_case(13, [1] * 20, np.arange(20), [11, 9], [64, 700], 32, 8, 128)
    ctx = make_ctx(c, groups=2)
    a, b = device_args(c), device_args(other)
    outs = []
    for _ in range(3):
        outs.append(ctx.prefix_attn(c["q"], c["kc"], c["vc"], **a))
        ctx.prefix_attn(other["q"], other["kc"], other["vc"], **b)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    check(c, outs[0], None)


def test_plan_in_select_is_not_used_for_the_own_parts_nor_left_stale():
    """The list that a selector leaves for dcut_verify_attn is another one, and outlives a shared-prefix call in between."""
    c = make_case(14, [3, 2, 4, 1], [40, 100, 7, 0], [4], [0], 8, 2, 128)
    ctx = make_ctx(c, max_gamma=3)
    ctx.enable_plan_in_select(True)
    conf = torch.full((4, 3), 0.9, device="cuda")
    ctx.set_cost_dense(np.linspace(1, 1.1, 20).astype(np.float32))
    z = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    a = device_args(c)
    sel = ctx.select(conf, z, z[:, 0].contiguous(), a["ctx_lens"])
    T = int(sel.cu_q[-1])
    q = torch.randn((T, 8, 128), device="cuda").to(torch.bfloat16)
    table = _i32(np.tile(np.arange(c["kc"].shape[0]), (4, 1)))[:, : a["block_table"].shape[1]].contiguous()
    want = ctx.verify_attn(q, c["kc"].nan_to_num(), c["vc"].nan_to_num(), table, a["ctx_lens"], sel.cu_q, T)
    ctx.prefix_attn(c["q"], c["kc"], c["vc"], **a)
    got = ctx.verify_attn(q, c["kc"].nan_to_num(), c["vc"].nan_to_num(), table, a["ctx_lens"], sel.cu_q, T)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_bad_page_is_reported():
    c = make_case(15, [2, 3], [5, 6], [2], [90], 8, 2, 128, poison=False)
    ctx = make_ctx(c)
    c["ptable"][0, 3] = c["kc"].shape[0]
    ctx.prefix_attn(c["q"], c["kc"], c["vc"], **device_args(c))
    assert ctx.poll_device_status() == 2


@pytest.mark.parametrize("what,code", [("short_context", 9), ("cover", 9), ("order", 9), ("long_prefix", 9), ("huge_prefix", 9), ("negative", 9),
                                       ("cu_q_past_cap", 7), ("cu_q_deep", 7), ("cu_q_empty", 7)])
def test_batches_that_break_the_contract_are_reported_and_left_alone(what, code):
    c = make_case(16, [2, 3, 1], [5, 6, 9], [2, 1], [90, 40], 8, 2, 128)
    ctx = make_ctx(c, max_gamma=3)
    if what == "short_context":
        c["ctx"][1] = 89
    elif what == "cover":
        c["cu_group"][-1] = 2
    elif what == "order":
        c["cu_group"][1] = 4
    elif what == "long_prefix":
        c["plens"][0] = 16 * c["ptable"].shape[1] + 1
    elif what == "huge_prefix":
        c["plens"][0] = 2 ** 31 - 1
    elif what == "negative":
        c["plens"][1] = -1
    elif what == "cu_q_past_cap":
        c["cu"][-1] = c["cap"] + 1
    elif what == "cu_q_deep":
        c["cu"][1] = 5
    else:
        c["cu"][1] = 0
    out = torch.full((c["cap"], 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.prefix_attn(c["q"], c["kc"], c["vc"], out=out, **device_args(c))
    assert ctx.poll_device_status() == code and bool((out == 7).all())


def test_not_enabled_and_too_many_groups_are_refused():
    from paper_2607_14647_b200 import binding
    c = make_case(17, [2, 3, 1], [5, 6, 9], [2, 1], [90, 40], 8, 2, 128)
    ctx = binding.Context(max_B=3, max_gamma=2, n_q_heads=8, n_kv_heads=2, head_dim=128, max_pages_per_req=64)
    for n in (0, 1):
        if n:
            ctx.enable_prefix_attn(n)
        with pytest.raises(binding.DcutError) as e:
            ctx.prefix_attn(c["q"], c["kc"], c["vc"], **device_args(c))
        assert e.value.status == binding.ECAPACITY
    ctx.enable_prefix_attn(2)
    check(c, *run(c, ctx))


def test_captured_and_replayed_with_other_contents():
    """A captured step serves later batches: cu_q, lengths and tables are read on the device at replay."""
    a = make_case(18, [5, 1, 17, 9], [5, 60, 9, 300], [3, 1], [190, 400], 8, 2, 128, cap=68, extra_pages=40)
    b = make_case(19, [17, 17, 2, 1], [50, 0, 90, 3], [2, 2], [260, 97], 8, 2, 128, cap=68, extra_pages=40)
    pool = max(a["kc"].shape[0], b["kc"].shape[0])
    cols, pcols = (max(a[t].shape[1], b[t].shape[1]) for t in ("table", "ptable"))
    for c in (a, b):
        for t, n in (("table", cols), ("ptable", pcols)):
            c[t] = np.pad(c[t], ((0, 0), (0, n - c[t].shape[1])))
        for t in ("kc", "vc"):
            c[t] = torch.cat([c[t], c[t][:1].expand(pool - c[t].shape[0], -1, -1, -1)]).contiguous()
    ctx = make_ctx(a, max_gamma=16)
    st = {k: a[k].clone() for k in ("q", "kc", "vc")}
    args = device_args(a)
    out, lse = torch.zeros((68, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((68, 8), device="cuda")
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        ctx.prefix_attn(st["q"], st["kc"], st["vc"], out=out, lse=lse, **args)
    for c in (a, b, a):
        other = device_args(c)
        for k in st:
            st[k].copy_(c[k])
        for k in ("block_table", "ctx_lens", "cu_q"):
            args[k].copy_(other[k])
        for x, y in zip(args["groups"].keep, other["groups"].keep):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert ctx.poll_device_status() == 0
        check(c, out, lse)


def test_two_contexts_on_two_streams():
    cases = [make_case(20 + i, [17] * 8, np.arange(8) * 20, [8], [1200], 32, 8, 128) for i in range(2)]
    ctxs = [make_ctx(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    args = [device_args(c) for c in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                outs[i].append(ctxs[i].prefix_attn(cases[i]["q"], cases[i]["kc"], cases[i]["vc"], **args[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert ctxs[i].poll_device_status() == 0
        assert all(torch.equal(o, outs[i][0]) for o in outs[i])
        check(cases[i], outs[i][0], None)


def poison_own_slots(c, k_value, v_value):
    """What lies behind a request's last position in its own pages."""
    group = np.repeat(np.arange(c["G"]), np.diff(c["cu_group"]))
    for r in range(c["B"]):
        end = int(c["ctx"][r] - c["plens"][group[r]] + c["counts"][r])
        if end % 16:
            page = int(c["table"][r, end // 16])
            c["kc"][page, :, end % 16:] = k_value
            c["vc"][page, :, end % 16:] = v_value


@pytest.mark.parametrize("value", [NAN, float("inf"), -float("inf"), 3.3e38])
@pytest.mark.parametrize("hq,hkv,d,deep", [(8, 8, 128, 1), (8, 2, 128, 17), (6, 2, 64, 9), (32, 4, 128, 17), (32, 2, 128, 9), (18, 2, 128, 16)])
def test_unwritten_slots_behind_a_request_hold_anything(hq, hkv, d, deep, value):
    """Warp-level tiles, tensor-memory tiles, their tails of up to 8 and 16 rows; long and short contexts."""
    rng = np.random.default_rng(hq + deep)
    counts = rng.integers(1, deep + 1, 20)
    counts[:3] = deep
    c = make_case(21, counts, np.concatenate([rng.integers(0, 100, 17), [1000, 2203, 4007]]), [11, 9], [70, 0], hq, hkv, d)
    ctx = make_ctx(c)
    clean, clean_lse = run(c, ctx)
    poison_own_slots(c, value, value)
    out, lse = run(c, ctx)
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)
    check(c, out, lse)


@pytest.mark.parametrize("hq,hkv,d,deep", [(8, 8, 128, 1), (8, 2, 64, 17), (32, 4, 128, 17), (32, 2, 128, 9)])
def test_verify_attn_with_unwritten_slots(hq, hkv, d, deep):
    rng = np.random.default_rng(hq + deep)
    counts = rng.integers(1, deep + 1, 12)
    counts[0] = deep
    c = make_case(22, counts, rng.integers(0, 3000, 12), [12], [0], hq, hkv, d)
    poison_own_slots(c, NAN, NAN)
    ctx = make_ctx(c)
    out = ctx.verify_attn(c["q"], c["kc"], c["vc"], _i32(c["table"]), _i32(c["ctx"]), _i32(c["cu"]), c["cap"])
    check(c, out, None)


def test_a_replayed_call_leaves_the_selector_s_list_alone():
    """The host cannot see a replay: the list that a selector left has to survive a captured shared-prefix call."""
    c = make_case(15, [3, 2, 4, 1], [40, 100, 7, 0], [3, 1], [33, 0], 8, 2, 128)
    ctx = make_ctx(c, max_gamma=3)
    ctx.enable_plan_in_select(True)
    ctx.set_cost_dense(np.linspace(1, 1.1, 20).astype(np.float32))
    conf, z, a = torch.full((4, 3), 0.9, device="cuda"), torch.zeros((4, 3), dtype=torch.int32, device="cuda"), device_args(c)
    bonus, out = z[:, 0].contiguous(), torch.zeros_like(c["q"])
    ctx.prefix_attn(c["q"], c["kc"], c["vc"], out=out, **a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.prefix_attn(c["q"], c["kc"], c["vc"], out=out, **a)
    kc, vc = c["kc"].nan_to_num(), c["vc"].nan_to_num()
    table = _i32(np.tile(np.arange(c["kc"].shape[0]), (4, 1)))[:, : a["block_table"].shape[1]].contiguous()
    sel = ctx.select(conf, z, bonus, a["ctx_lens"])
    T = int(sel.cu_q[-1])
    q = torch.randn((T, 8, 128), device="cuda").to(torch.bfloat16)
    want = ctx.verify_attn(q, kc, vc, table, a["ctx_lens"], sel.cu_q, T).clone()
    sel = ctx.select(conf, z, bonus, a["ctx_lens"])
    graph.replay()
    got = ctx.verify_attn(q, kc, vc, table, a["ctx_lens"], sel.cu_q, T)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("B,size", [(4096, 2), (4097, 1), (6000, 100)])
def test_thousands_of_requests(B, size):
    """More requests and groups than the plan keeps in shared memory, and the most that it does."""
    rng = np.random.default_rng(B)
    sizes = [size] * (B // size) + ([B % size] if B % size else [])
    c = make_case(B, rng.integers(1, 3, B), rng.integers(0, 20, B), sizes, rng.integers(0, 40, len(sizes)), 1, 1, 64)
    check(c, *run(c))


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (2, 2, 64), (9, 1, 128)])
@pytest.mark.parametrize("longest", [64, 200, 600])
def test_many_short_items_per_segment(longest, hq, hkv, d):
    """Several items behind one another in every CTA: with no block, one (the second team has none), a few; cut and whole."""
    rng = np.random.default_rng(longest + hq)
    sizes = rng.integers(0, 4, 700)
    B = int(sizes.sum())
    plens = rng.integers(0, longest + 1, 700)
    c = make_case(longest, rng.integers(1, 4, B), rng.integers(0, 40, B), sizes, plens, hq, hkv, d)
    check(c, *run(c))


def test_pages_behind_two_to_the_31_elements():
    """The same pages at the end of a cache of more than 2^31 elements give the same bits."""
    c = make_case(31, [3, 1, 9], [40, 7, 300], [3], [150], 8, 8, 128)
    ctx = make_ctx(c)
    want, want_lse = run(c, ctx)
    pool, shift = c["kc"].shape[0], 2 ** 31 // (8 * 16 * 128) + 5
    for n in ("kc", "vc"):
        big = torch.empty((shift + pool, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
        big[:2] = NAN
        big[shift:] = c[n]
        c[n] = big
    c["table"], c["ptable"] = c["table"] + shift, c["ptable"] + shift
    c["table"][c["table"] > shift + pool] = 1 << 30
    out, lse = run(c, ctx)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (2, 2, 64)])
def test_odd_singles_before_other_items(hq, hkv, d):
    """Items of one tile with an odd number of blocks behind one another in a CTA, and before items of two tiles: a slot of
    the ring changes hands between the teams.  The same bits every time."""
    rng = np.random.default_rng(hq)
    sizes = rng.integers(1, 4, 300)
    sizes[::7] = 70                                    # more than a tile of tokens (64 or 128), at three rows each
    B = int(sizes.sum())
    plens = 64 * rng.choice([1, 3, 5, 7], 300) - rng.integers(0, 20, 300)
    c = make_case(32, rng.integers(1, 4, B), rng.integers(0, 20, B), sizes, plens, hq, hkv, d)
    ctx = make_ctx(c)
    out, lse = run(c, ctx)
    check(c, out, lse)
    for _ in range(5):
        again, lse2 = run(c, ctx)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("request_", [0, 1, 2])
@pytest.mark.parametrize("excess", [1, 16, 100000, None])
def test_own_positions_behind_the_block_table_are_reported(request_, excess):
    """The last row's position has to lie in the request's row of the block table; where it just does, nothing is reported."""
    c = make_case(33, [2, 3, 1], [5, 6, 9], [2, 1], [90, 40], 8, 2, 128)
    ctx = make_ctx(c, max_gamma=3)
    plen = c["plens"][0 if request_ < 2 else 1]
    c["ctx"][request_] = 2 ** 31 - 1 if excess is None else plen + 16 * c["table"].shape[1] - c["counts"][request_] + excess
    out = torch.full((c["cap"], 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.prefix_attn(c["q"], c["kc"], c["vc"], out=out, **device_args(c))
    assert ctx.poll_device_status() == 9 and bool((out == 7).all())


def test_own_positions_may_fill_the_block_table():
    c = make_case(34, [2, 3, 1], [16 * 4 - 2, 16 * 4 - 3, 16 * 4 - 1], [2, 1], [90, 40], 8, 2, 128)
    c["table"] = np.ascontiguousarray(c["table"][:, :4])
    check(c, *run(c))


# ------------------------------------------------------------------------------------- scores that are no numbers, where they are seen

def assert_not_numbers_where_the_formula_has_them(c, out, lse, clean, clean_lse):
    """NaN in exactly the rows (and, for V, columns) that the formula gives it in; what the planted key does not touch keeps its bits.
    A row to which the planted key is at minus infinity differs from the clean one by that key alone: the clean scores' bound."""
    d = c["d"]
    args = (c["table"], c["ctx"], c["cu"], c["cu_group"], c["plens"], c["ptable"], d ** -0.5)
    q = bf16_values(c["q"])
    with np.errstate(invalid="ignore"):
        want, want_lse, A, _ = plain(q, c["kc_plain"], c["vc_plain"], *args)
    _, _, _, qk = plain(q, c["kc_clean"], c["vc_clean"], *args)
    T = c["T"]
    want, want_lse, A, E = want[:T], want_lse[:T], A[:T], d * 2.0 ** -23 * qk[:T]
    got, got_lse = bf16_values(out)[:T], lse.cpu().numpy().astype(np.float64)[:T]
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), (np.isfinite(got) != np.isfinite(want)).sum()
    assert np.array_equal(np.isnan(got_lse), np.isnan(want_lse)), (np.isnan(got_lse) != np.isnan(want_lse)).sum()
    bad = ~np.isfinite(want)
    assert bad.any() or not np.isfinite(c["planted"])
    with np.errstate(invalid="ignore"):
        lim = 2.0 ** -8 * (np.abs(want) + A) + (2 * E[..., None] + 2.0 ** -15) * A
        assert (np.abs(got - want) <= lim)[~bad].all()
        assert (np.abs(got_lse - want_lse) <= E + 2.0 ** -18 + 2.0 ** -21 * np.abs(want_lse))[~np.isnan(want_lse)].all()
    same = c["untouched"][:T]
    assert torch.equal(out[:T][same], clean[:T][same]) and torch.equal(lse[:T][same], clean_lse[:T][same])
    return bad


def plant(c, cache, page, slot, value, head=0, element=3):
    c[cache][int(page), head, int(slot), element] = value
    c[cache + "_plain"][int(page), head, int(slot), element] = value
    c["planted"] = value


def planted_case(*args, **kw):
    c = make_case(*args, poison=False, **kw)
    c["kc_clean"], c["vc_clean"] = c["kc_plain"].copy(), c["vc_plain"].copy()
    group = np.repeat(np.arange(c["G"]), np.diff(c["cu_group"]))
    c["group_of_row"], c["req_of_row"] = np.repeat(group, c["counts"]), np.repeat(np.arange(c["B"]), c["counts"])
    return c


# one tile or two per group; one long prefix that is cut over the SMs, or more whole items than SMs
SHARED = {"cut_single": ([3, 1, 5], [3], [1000], 8, 2), "cut_dual": ([17, 9, 4], [3], [2500], 32, 4), "whole_single": ([2, 1] * 150, [1] * 300, [130] * 300, 8, 2),
          "whole_dual": ([17, 17] * 60, [2] * 60, [200] * 60, 16, 2), "one_block": ([2], [1], [9], 4, 2)}


@pytest.mark.parametrize("value", [NAN, float("inf")])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("shape", sorted(SHARED))
def test_a_key_of_a_prefix_that_is_no_number_shows(shape, d, value):
    counts, sizes, plens, hq, hkv = SHARED[shape]
    c = planted_case(41, counts, np.arange(len(counts)) % 30, sizes, plens, hq, hkv, d)
    ctx = make_ctx(c)
    clean, clean_lse = run(c, ctx)
    kc = c["kc"].clone()
    P = plens[0]
    for j in sorted({0, P // 2, P - 1}):
        c["kc"].copy_(kc)
        c["kc_plain"] = c["kc_clean"].copy()
        plant(c, "kc", c["ptable"][0, j // 16], j % 16, value, head=hkv - 1)
        c["untouched"] = torch.tensor((c["group_of_row"] > 0)[:, None] | (np.arange(hq) < hq - hq // hkv), device="cuda")
        out, lse = run(c, ctx)
        assert_not_numbers_where_the_formula_has_them(c, out, lse, clean, clean_lse)


@pytest.mark.parametrize("value", [NAN, float("inf")])
@pytest.mark.parametrize("shape", sorted(SHARED))
def test_a_value_of_a_prefix_that_is_no_number_shows_in_its_column(shape, value):
    counts, sizes, plens, hq, hkv = SHARED[shape]
    c = planted_case(42, counts, np.arange(len(counts)) % 30, sizes, plens, hq, hkv, 128)
    ctx = make_ctx(c)
    clean, clean_lse = run(c, ctx)
    plant(c, "vc", c["ptable"][0, 0], 5, value)
    c["untouched"] = torch.tensor((c["group_of_row"] > 0)[:, None] | (np.arange(hq) >= hq // hkv), device="cuda")
    out, lse = run(c, ctx)
    bad = assert_not_numbers_where_the_formula_has_them(c, out, lse, clean, clean_lse)
    assert torch.equal(lse, clean_lse) and bad[..., 3].sum() == bad.sum()


@pytest.mark.parametrize("value", [NAN, float("inf")])
@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("hq,hkv,d,deep", [(8, 8, 128, 1), (8, 2, 64, 17), (8, 2, 128, 17), (32, 4, 128, 17), (32, 2, 128, 9), (18, 2, 128, 16)])
def test_a_key_of_a_request_that_is_no_number_shows(hq, hkv, d, deep, prefix, value):
    """Own keys: warp-level tiles, tensor-memory tiles and their tails, whole and cut; the last key may be all that a team of
    softmax warps sees.  dcut_verify_attn, which shares that path, alike."""
    counts = [deep, deep, 1, max(1, deep - 4)] * 3
    own = [64 - deep + 1, 0, 64, 127, 200, 1000, 4007, 448, 64, 7, 2203, 128]
    c = planted_case(43, counts, own, [len(counts)], [prefix], hq, hkv, d)
    ctx = make_ctx(c)
    clean, clean_lse = run(c, ctx)
    for r, back in ((0, 0), (2, 0), (5, 500), (6, 0), (6, 3000), (7, 0), (10, 1)):
        j = int(own[r] + counts[r] - 1 - back)                          # back 0: the request's last token, which one row sees
        if j < 0:
            continue
        plant(c, "kc", c["table"][r, j // 16], j % 16, value)
    touched = np.isin(c["req_of_row"], [0, 2, 5, 6, 7, 10])
    c["untouched"] = torch.tensor(~touched[:, None] | (np.arange(hq) >= hq // hkv), device="cuda")
    out, lse = run(c, ctx)
    assert_not_numbers_where_the_formula_has_them(c, out, lse, clean, clean_lse)
    if prefix == 0:
        lse2 = torch.empty_like(lse)
        a = device_args(c)
        out2 = ctx.verify_attn(c["q"], c["kc"], c["vc"], a["block_table"], a["ctx_lens"], a["cu_q"], c["cap"], lse=lse2)
        torch.cuda.synchronize()
        assert_not_numbers_where_the_formula_has_them(c, out2, lse2, out2, lse2)


@pytest.mark.parametrize("counts,own,sizes,plens,hq,hkv,d", [([1] * 16, list(range(0, 160, 10)), [16], [512], 32, 8, 128), ([17] * 8 + [3] * 4, [30] * 12, [7, 5], [160, 2048], 16, 2, 128),
                                                           ([5, 9, 1], [0, 40, 700], [3], [1008], 8, 8, 64)])
def test_agrees_with_verify_attn_where_the_prefix_s_pages_are_joined_to_every_request_s(counts, own, sizes, plens, hq, hkv, d):
    c = make_case(44, counts, own, sizes, plens, hq, hkv, d)
    group = np.repeat(np.arange(c["G"]), sizes)
    joined = np.full((c["B"], max(plens) // 16 + c["table"].shape[1]), -1)
    for r in range(c["B"]):
        n = plens[group[r]] // 16
        joined[r, :n] = c["ptable"][group[r], :n]
        joined[r, n:n + c["table"].shape[1]] = c["table"][r]
    ctx = make_ctx(c)
    out, lse = run(c, ctx)
    from paper_2607_14647_b200 import binding
    whole = binding.Context(max_B=c["B"], max_gamma=max(1, max(counts) - 1), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_pages_per_req=joined.shape[1])
    lse2 = torch.empty_like(lse)
    out2 = whole.verify_attn(c["q"], c["kc"], c["vc"], _i32(joined), _i32(c["ctx"]), _i32(c["cu"]), c["cap"], lse=lse2)
    torch.cuda.synchronize()
    assert whole.poll_device_status() == 0
    check(c, out, lse)
    check(c, out2, lse2)
