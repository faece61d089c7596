"""Cases that measure three operators of a verification step: the rotary append to the paged cache, attention behind a
shared prefix, and the linear layer with its epilogue.

`own` False: their plain forms, elementary torch operations in 32 bits.  `own` True: the calls of `binding.Context`.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1e-6
THETA = 1.0e6
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_contexts = {}


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    def append(name, **kw):
        return dict(dict(op="append", name=name, heads_q=32, heads_kv=8, dim=128, rotary=128, interleaved=False, norm=False,
                         fused=True, prefix=0), **kw)

    def prefix(name, **kw):
        return dict(dict(op="prefix", name=name, heads_q=32, heads_kv=8, dim=128, groups=1, bare=False), **kw)

    def linear(name, **kw):
        return dict(dict(op="linear", name=name, act="none", bias=True, gated=False, residual=False), **kw)

    return [
        # the new token of each request of a small batch: one launch, latency counts
        append("append_decode_b16", B=16, tokens=16, deep=1, cap=16, ctx_lo=1024, ctx_hi=4096, fused=False),
        # a pruned verification batch behind a system prompt, far positions, a target with q/k norm
        append("append_verify_b64", B=64, tokens=603, deep=17, cap=1088, ctx_lo=2048, ctx_hi=131072, prefix=2048, norm=True),
        # three prompts at once, interleaved pairs on half of the head
        append("append_prompt_8191", B=3, tokens=8191, deep=4000, cap=8191, ctx_lo=0, ctx_hi=999, heads_q=64, rotary=64,
               interleaved=True),
        # single tokens behind one prompt
        prefix("prefix_decode_b16", B=16, tokens=16, deep=1, prefix=2048, own_lo=64, own_hi=512),
        # the pruned batch of 64 behind a prompt that ends inside a page
        prefix("prefix_verify_b64", B=64, tokens=603, deep=17, prefix=4099, own_lo=512, own_hi=2048),
        # three tenants, one of them without a shared prompt, wide query groups
        prefix("prefix_groups_b48", B=48, tokens=517, deep=17, heads_q=64, groups=3, bare=True, prefix=6000, own_lo=0, own_hi=1500),
        # a small model: head size 64, a key head per query head
        prefix("prefix_dim64_b24", B=24, tokens=130, deep=17, heads_q=16, heads_kv=16, dim=64, prefix=1023, own_lo=1, own_hi=300),
        # a full batch at full depth behind a long prompt: the shared part is nearly all of the work
        prefix("prefix_long_b128", B=128, tokens=2176, deep=17, prefix=8192, own_lo=128, own_hi=512),
        # the QKV projection (32 + 2 x 8 heads of 128) of a few tokens: the weight is what moves
        linear("linear_decode_qkv", tokens=7, cap=16, k=4096, n=6144),
        # nothing divides anything, rows padded
        linear("linear_odd_relu", tokens=333, cap=512, k=1003, n=2051, act="relu", residual=True),
        # a two-matrix MLP's first half at full depth
        linear("linear_gelu_t1088", tokens=1088, cap=1088, k=4096, n=12288, act="gelu_tanh"),
        # a gated projection added to the residual stream
        linear("linear_gated_t603", tokens=603, cap=1088, k=4096, n=4096, act="silu", gated=True, residual=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "prefix", "linear"))
    if op == "linear":
        tokens = _log(rng, 1, 1088)
        gated = rng.random() < 0.3
        return dict(op=op, tokens=tokens, cap=tokens + rng.randint(0, 200), k=_log(rng, 17, 4096), n=_log(rng, 9, 6000 if gated else 12000),
                    act=rng.choice(ACTS), bias=rng.random() < 0.7, gated=gated, residual=rng.random() < 0.5)
    dim = rng.choice((64, 128, 128))
    kv, per = rng.choice(((8, 4), (8, 8), (2, 6), (16, 1), (4, 5), (1, 4)))
    if op == "append":
        B = _log(rng, 1, 128)
        deep = _log(rng, 1, max(1, 8191 // B))
        tokens = rng.randint(B, B * deep)
        prefix = rng.choice((0, 0, 100, 2048))
        lo = prefix + _log(rng, 1, 3000)
        return dict(op=op, B=B, tokens=tokens, deep=deep, cap=tokens + rng.randint(0, 50), heads_q=kv * per, heads_kv=kv, dim=dim,
                    rotary=rng.choice((16, 32, 64, dim)), interleaved=rng.random() < 0.5, norm=rng.random() < 0.5,
                    fused=rng.random() < 0.5, prefix=prefix, ctx_lo=lo, ctx_hi=lo + _log(rng, 1, 200000))
    B = _log(rng, 1, 64)
    deep = rng.choice((1, 4, 9, 17))
    groups = rng.randint(1, min(B, 4))
    lo = rng.randint(0, 200)
    return dict(op=op, B=B, tokens=rng.randint(B, B * deep), deep=deep, heads_q=kv * per, heads_kv=kv, dim=dim, groups=groups,
                bare=groups > 1 and rng.random() < 0.5, prefix=_log(rng, 1, 8192), own_lo=lo, own_hi=lo + _log(rng, 1, 1500))


# ------------------------------------------------------------------------------------------- what follows from the case

def _spread(lo, hi, n):
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _share(total, parts):
    return [total * (i + 1) // parts - total * i // parts for i in range(parts)]


def _prefix_lens(c):
    G = c["groups"]
    lens = [c["prefix"] * (G - g) // G for g in range(G)]
    if c["bare"]:
        lens[-1] = 0
    return lens


def _group_tokens(c):
    """Tokens of each group: every request one, the rest by the groups' sizes."""
    sizes = _share(c["B"], c["groups"])
    edges = np.cumsum([0] + sizes)
    extra = c["tokens"] - c["B"]
    return sizes, [s + extra * int(e1) // c["B"] - extra * int(e0) // c["B"] for s, e0, e1 in zip(sizes, edges[:-1], edges[1:])]


def work(c):
    if c["op"] == "linear":
        t, k, n, g = c["tokens"], c["k"], c["n"], 2 if c["gated"] else 1
        return {"bytes": 2 * (t * k + g * n * k + t * n * (2 if c["residual"] else 1) + (g * n if c["bias"] else 0)), "flops": 2 * g * t * n * k}
    hq, hkv, d, t = c["heads_q"], c["heads_kv"], c["dim"], c["tokens"]
    if c["op"] == "append":
        return {"bytes": 4 * t * (hq + 2 * hkv) * d, "flops": 6 * t * (hq + hkv) * c["rotary"]}
    lens, (_, tokens) = _prefix_lens(c), _group_tokens(c)
    own_keys = sum(_spread(c["own_lo"], c["own_hi"], c["B"]))
    return {"bytes": 4 * hkv * d * (sum(lens) + own_keys + t) + 4 * t * hq * d + 4 * t * hq,
            "flops": 4 * hq * d * (sum(p * n for p, n in zip(lens, tokens)) + t * own_keys // c["B"])}


# -------------------------------------------------------------------------------------------------------------- prepare

def _counts(rng, B, tokens, deep):
    """Tokens per request, 1 .. deep each, `tokens` in all."""
    picked = rng.permutation(B * (deep - 1))[: tokens - B]
    return 1 + np.bincount(picked % B, minlength=B)


def _int(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _context(**limits):
    """A serving process makes one context for its model and keeps it."""
    key = tuple(sorted(limits.items()))
    if key not in _contexts:
        from paper_2607_14647_b200 import binding
        _contexts[key] = binding.Context(**limits)
    return _contexts[key]


def _context_for(c):
    g = c["deep"] - 1 if c["op"] == "prefix" else 1
    return _context(max_B=c["B"], max_gamma=max(1, g), n_q_heads=c["heads_q"], n_kv_heads=c["heads_kv"], head_dim=c["dim"],
                    max_pages_per_req=16384)


def prepare(c, seed):
    rng = np.random.default_rng([seed, 1])
    gen = torch.Generator("cuda").manual_seed(seed)
    return {"append": _prepare_append, "prefix": _prepare_prefix, "linear": _prepare_linear}[c["op"]](c, rng, gen)


def _prepare_append(c, rng, gen):
    B, T, hq, hkv, d = c["B"], c["tokens"], c["heads_q"], c["heads_kv"], c["dim"]
    counts = _counts(rng, B, T, c["deep"])
    ctx = rng.permutation(_spread(c["ctx_lo"], c["ctx_hi"], B))
    req = np.repeat(np.arange(B), counts)
    cu = np.concatenate([[0], np.cumsum(counts)])
    pos = ctx[req] + np.arange(T) - cu[req]
    page_of = (pos - c["prefix"]) // PAGE
    touched = np.unique(req * (1 << 32) + page_of)
    pool = min(T, T // PAGE + 2 * B) + 64  # room for every page that is touched, however the tokens fall
    table = rng.integers(0, pool, (B, int(page_of.max()) + 1))
    table[touched >> 32, touched & 0xffffffff] = rng.permutation(pool)[: len(touched)]
    cap = c["cap"]
    if c["fused"]:  # rows of a QKV projection
        x = _normal(gen, cap, hq + 2 * hkv, d)
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    else:
        q, k, v = _normal(gen, cap, hq, d), _normal(gen, cap, hkv, d), _normal(gen, cap, hkv, d)
    s = dict(c=c, T=T, q=q, k=k, v=v, table=_int(table), req=_int(np.concatenate([req, np.full(cap - T, -1)])),
             pos=_int(np.concatenate([pos, np.full(cap - T, -1)])), cu=_int(cu),
             freq=torch.tensor([THETA ** (-2.0 * e / c["rotary"]) for e in range(c["rotary"] // 2)], dtype=torch.float64, device="cuda"),
             q_gain=1 + 0.1 * _normal(gen, d) if c["norm"] else None, k_gain=1 + 0.1 * _normal(gen, d) if c["norm"] else None,
             k_cache=_normal(gen, pool, hkv, PAGE, d), v_cache=_normal(gen, pool, hkv, PAGE, d),
             q_out=torch.zeros((cap, hq, d), dtype=torch.bfloat16, device="cuda"))
    if own:
        from paper_2607_14647_b200 import binding
        s["ctx"] = _context_for(c)
        s["shared"] = binding.PrefixGroups(_int([0, B]), _int([c["prefix"]]), _int(np.zeros((1, c["prefix"] // PAGE + 1)))) if c["prefix"] else None
    return s


def _prepare_prefix(c, rng, gen):
    B, T, hq, hkv, d = c["B"], c["tokens"], c["heads_q"], c["heads_kv"], c["dim"]
    lens, (sizes, tokens) = _prefix_lens(c), _group_tokens(c)
    counts = np.concatenate([_counts(rng, n, t, c["deep"]) for n, t in zip(sizes, tokens)])
    own_len = rng.permutation(_spread(c["own_lo"], c["own_hi"], B))
    group = np.repeat(np.arange(c["groups"]), sizes)
    plen = np.array(lens)[group]
    own_pages = -(-(own_len + counts) // PAGE)
    shared_pages = [-(-p // PAGE) for p in lens]
    pool = int(own_pages.sum()) + sum(shared_pages) + 1
    free = rng.permutation(pool)
    table, shared = np.zeros((B, int(own_pages.max()))), np.zeros((c["groups"], max(1, max(shared_pages))))
    at = 0
    for rows, need in ((table, own_pages), (shared, shared_pages)):
        for i, n in enumerate(need):
            rows[i, :n] = free[at:at + n]
            at += n
    s = dict(c=c, T=T, q=1.5 * _normal(gen, T, hq, d), k_cache=_normal(gen, pool, hkv, PAGE, d), v_cache=_normal(gen, pool, hkv, PAGE, d),
             table=_int(table), shared_table=_int(shared), counts=_int(counts), group=_int(group), plen=_int(plen), ctx_lens=_int(plen + own_len),
             cu=_int(np.concatenate([[0], np.cumsum(counts)])), longest=int((plen + own_len + counts).max()),
             out=torch.zeros((T, hq, d), dtype=torch.bfloat16, device="cuda"), lse=torch.zeros((T, hq), dtype=torch.float32, device="cuda"))
    if own:
        from paper_2607_14647_b200 import binding
        s["ctx"] = _context_for(c)
        s["ctx"].enable_prefix_attn(c["groups"])
        s["shared"] = binding.PrefixGroups(_int(np.concatenate([[0], np.cumsum(sizes)])), _int(lens), s["shared_table"])
    return s


def _prepare_linear(c, rng, gen):
    k, n, cap = c["k"], c["n"], c["cap"]
    ld = -(-k // 8) * 8  # rows start on 16 bytes
    a = _normal(gen, cap, ld)[:, :k]

    def weight():
        return (_normal(gen, n, ld) / math.sqrt(k))[:, :k]

    def bias():
        return _normal(gen, n) if c["bias"] else None

    s = dict(c=c, T=c["tokens"], a=a, w=weight(), bias=bias(), w2=weight() if c["gated"] else None, bias2=bias() if c["gated"] else None,
             residual=_normal(gen, cap, n) if c["residual"] else None, cu=_int([0, c["tokens"]]),
             out=torch.zeros((cap, n), dtype=torch.bfloat16, device="cuda"))
    if own:
        s["ctx"] = _context(max_B=64, max_gamma=16, n_q_heads=32, n_kv_heads=8, head_dim=128, max_pages_per_req=1024)
    return s


# ------------------------------------------------------------------------------------------------------------------ run

def run(s):
    return {"append": _run_append, "prefix": _run_prefix, "linear": _run_linear}[s["c"]["op"]](s)


def _run_append(s):
    c = s["c"]
    if own:
        s["ctx"].rope_append(s["q"], s["k"], s["v"], s["freq"], s["k_cache"], s["v_cache"], s["table"], s["req"], s["pos"], c["cap"],
                             cu_q=s["cu"], interleaved=c["interleaved"], q_gain=s["q_gain"], k_gain=s["k_gain"], rms_eps=EPS,
                             groups=s["shared"], q_out=s["q_out"])
        return s["q_out"], s["k_cache"], s["v_cache"]
    T, r = s["T"], c["rotary"]
    pos = s["pos"][:T].long()
    angle = pos.double()[:, None] * s["freq"]  # far positions: 32 bits would lose the angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotated(x, gain):
        x = x[:T].float()
        if gain is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()
        y = x.clone()
        a, b = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., b] * cos + x[..., a] * sin
        return y.to(torch.bfloat16)

    s["q_out"][:T] = rotated(s["q"], s["q_gain"])
    slot = pos - c["prefix"]
    page = s["table"][s["req"][:T].long(), slot // PAGE].long()
    s["k_cache"][page, :, slot % PAGE] = rotated(s["k"], s["k_gain"])
    s["v_cache"][page, :, slot % PAGE] = s["v"][:T]
    return s["q_out"], s["k_cache"], s["v_cache"]


def _run_prefix(s):
    c = s["c"]
    if own:
        s["ctx"].prefix_attn(s["q"], s["k_cache"], s["v_cache"], s["table"], s["ctx_lens"], s["cu"], s["T"], s["shared"], out=s["out"], lse=s["lse"])
        return s["out"], s["lse"]
    B, hq, hkv, d, dev = c["B"], c["heads_q"], c["heads_kv"], c["dim"], s["q"].device
    j = torch.arange(s["longest"], device=dev)
    plen, last = s["plen"].long()[:, None], s["ctx_lens"].long()[:, None] + s["counts"].long()[:, None] - 1
    at = torch.where(j < plen, j, (j - plen).clamp(min=0))
    at = torch.minimum(at, torch.where(j < plen, plen - 1, last - plen))  # behind the last key: any page that exists, masked below
    page = torch.where(j < plen, s["shared_table"][s["group"].long()[:, None], (at // PAGE).clamp(max=s["shared_table"].shape[1] - 1)],
                       s["table"][torch.arange(B, device=dev)[:, None], (at // PAGE).clamp(max=s["table"].shape[1] - 1)]).long()
    k = s["k_cache"][page, :, at % PAGE].float()  # [B, keys, kv heads, dim]
    v = s["v_cache"][page, :, at % PAGE].float()
    t = torch.arange(c["deep"], device=dev)
    row = (s["cu"].long()[:-1, None] + t).clamp(max=s["T"] - 1)
    live = t < s["counts"].long()[:, None]
    q = s["q"][row].float().reshape(B, c["deep"], hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(d)
    seen = (j <= s["ctx_lens"].long()[:, None, None] + t[:, None])[:, None, :, None].expand(B, 1, c["deep"], hq // hkv, s["longest"])
    score = score.masked_fill(~seen.reshape(B, 1, -1, s["longest"]), -math.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - top).exp()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v.permute(0, 2, 1, 3)) / total
    lse = top + total.log()
    o = o.reshape(B, hkv, c["deep"], hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, c["deep"], hq, d)
    lse = lse.reshape(B, hkv, c["deep"], hq // hkv).permute(0, 2, 1, 3).reshape(B, c["deep"], hq)
    s["out"][row[live]] = o[live].to(torch.bfloat16)
    s["lse"][row[live]] = lse[live]
    return s["out"], s["lse"]


def _activated(x, act):
    if act == "relu":
        return x.clamp(min=0)
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    if act == "silu":
        return x / (1 + torch.exp(-x))
    return x


def _run_linear(s):
    c = s["c"]
    if own:
        s["ctx"].linear(s["a"], s["w"], s["cu"], c["cap"], out=s["out"], bias=s["bias"], act=c["act"], w2=s["w2"], bias2=s["bias2"],
                        residual=s["residual"])
        return s["out"]
    T = s["T"]
    a = s["a"][:T].float()

    def product(w, bias):
        y = torch.matmul(a, w.float().t())
        return y if bias is None else y + bias.float()

    y = _activated(product(s["w"], s["bias"]), c["act"])
    if c["gated"]:
        y = y * product(s["w2"], s["bias2"])
    if c["residual"]:
        y = y + s["residual"][:T].float()
    s["out"][:T] = y.to(torch.bfloat16)
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------- exact

def exact(c, seed):
    """The operators' definitions, request by request, in 64 bits."""
    s = prepare(c, seed)
    if c["op"] == "linear":
        T, x = c["tokens"], s["a"].double()
        y = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for i in range(0, T, 256):
            rows = slice(i, min(T, i + 256))
            z = x[rows] @ s["w"].double().T
            if s["bias"] is not None:
                z += s["bias"].double()
            if c["act"] == "relu":
                z = torch.where(z > 0, z, 0.0)
            elif c["act"] == "gelu":
                z = z * torch.special.ndtr(z)
            elif c["act"] == "gelu_tanh":  # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
                z = z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
            elif c["act"] == "silu":
                z = z * torch.sigmoid(z)
            if c["gated"]:
                up = x[rows] @ s["w2"].double().T
                z = z * (up if s["bias2"] is None else up + s["bias2"].double())
            y[rows] = z if s["residual"] is None else z + s["residual"][rows].double()
        return y
    cu = s["cu"].tolist()
    table = s["table"].cpu().numpy()
    hq, hkv, d = c["heads_q"], c["heads_kv"], c["dim"]
    if c["op"] == "append":
        r, T = c["rotary"], c["tokens"]
        outs = [x.double() for x in (s["q_out"], s["k_cache"], s["v_cache"])]
        rows = []
        for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
            x = x[:T].double()
            if gain is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * gain.double()
            e = torch.arange(r // 2, device="cuda")
            first, second = (2 * e, 2 * e + 1) if c["interleaved"] else (e, e + r // 2)
            z = torch.polar(torch.ones(T, 1, r // 2, dtype=torch.float64, device="cuda"), (s["pos"][:T].double()[:, None] * s["freq"])[:, None, :])
            z = torch.complex(x[..., first], x[..., second]) * z
            x[..., first], x[..., second] = z.real, z.imag
            rows.append(x)
        outs[0][:T] = rows[0]
        pos = s["pos"].tolist()
        for i in range(c["B"]):
            a = 0
            while a < cu[i + 1] - cu[i]:  # the run of tokens that lies in one page
                slot = pos[cu[i] + a] - c["prefix"]
                n = min(PAGE - slot % PAGE, cu[i + 1] - cu[i] - a)
                page, to, at = int(table[i, slot // PAGE]), slice(slot % PAGE, slot % PAGE + n), slice(cu[i] + a, cu[i] + a + n)
                outs[1][page, :, to] = rows[1][at].transpose(0, 1)
                outs[2][page, :, to] = s["v"][at].double().transpose(0, 1)
                a += n
        return tuple(outs)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    shared = s["shared_table"]
    for i in range(c["B"]):
        p, ctx, n = int(s["plen"][i]), int(s["ctx_lens"][i]), cu[i + 1] - cu[i]

        def keys(cache):
            a = cache[shared[int(s["group"][i]), : -(-p // PAGE)].long()].transpose(1, 2).reshape(-1, hkv, d)[:p]
            m = ctx - p + n
            b = cache[s["table"][i, : -(-m // PAGE)].long()].transpose(1, 2).reshape(-1, hkv, d)[:m]
            return torch.cat([a, b]).double()

        k, v = keys(s["k_cache"]), keys(s["v_cache"])
        q = s["q"][cu[i]:cu[i + 1]].double().reshape(n, hkv, hq // hkv, d)
        z = torch.einsum("nhgd,jhd->nhgj", q, k) * d ** -0.5
        hidden = torch.arange(p + ctx - p + n, device="cuda")[None, :] > ctx + torch.arange(n, device="cuda")[:, None]
        z[hidden[:, None, None, :].expand_as(z)] = -math.inf
        out[cu[i]:cu[i + 1]] = torch.einsum("nhgj,jhd->nhgd", torch.softmax(z, -1), v).reshape(n, hq, d)
        lse[cu[i]:cu[i + 1]] = torch.logsumexp(z, -1).reshape(n, hq)
    return out, lse
