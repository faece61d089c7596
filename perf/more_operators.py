"""Cases that measure three operators of a target model held in 8 bits whose requests carry adapters: the RMS norm with the
residual's addition and an 8-bit output, the linear layer on 8-bit operands, and the requests' low-rank adapters.

`own` False: their plain forms, elementary torch operations in 32 bits.  `own` True: the calls of `binding.Context`.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
LEAST = 2.0 ** -100      # a row's largest value counts as at least this
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_contexts = {}


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    def norm(name, **kw):
        return dict(dict(op="norm", name=name, width=4096, normed=True, residual=True, bf16=False, fp8=True, pad=0), **kw)

    def linear(name, **kw):
        return dict(dict(op="linear8", name=name, act="none", bias=False, gated=False, residual=False), **kw)

    def lora(name, **kw):
        return dict(dict(op="lora", name=name, k=4096, act="none", gated=False, none=True), **kw)

    return [
        # the residual stream of a small decode batch on its way to an 8-bit projection: latency counts
        norm("norm_decode_b16", tokens=16, cap=16),
        # a pruned verification batch: 8-bit rows for the shared projection, bf16 rows for the adapters
        norm("norm_verify_t603", tokens=603, cap=1088, bf16=True),
        # prompts: the plain residual norm at length
        norm("norm_prompt_8191", tokens=8191, cap=8191, bf16=True),
        # the MLP's activation before its 8-bit down projection: no norm, wide rows
        norm("quant_mlp_t1088", tokens=1088, cap=1088, width=12288, normed=False, residual=False),
        # the QKV projection (32 + 2 x 8 heads of 128) of a few tokens: the weight is what moves
        linear("linear8_decode_qkv", tokens=7, cap=16, k=4096, n=6144, bias=True),
        # nothing divides anything
        linear("linear8_odd_relu", tokens=333, cap=512, k=1003, n=2051, act="relu", bias=True, residual=True),
        # gate and up projection of a verification batch at full depth
        linear("linear8_gated_t1088", tokens=1088, cap=1088, k=4096, n=12288, act="silu", gated=True),
        # the down projection of three prompts, onto the residual stream
        linear("linear8_prompt_8191", tokens=8191, cap=8191, k=12288, n=4096, residual=True),
        # the new token of each request, an adapter each, on q, k and v
        lora("lora_decode_b16", B=16, tokens=16, cap=16, adapters=16, rank=16, ends="4096,5120,6144"),
        # a pruned verification batch over 24 tenants, on the output projection
        lora("lora_verify_b64", B=64, tokens=603, cap=1088, adapters=24, rank=16, ends="4096"),
        # gate and up projection at full depth: the adapters join ahead of the activation
        lora("lora_gated_t1088", B=64, tokens=1088, cap=1088, adapters=8, rank=64, ends="12288,24576", act="silu", gated=True),
        # three prompts, each its own adapter
        lora("lora_prompt_8191", B=3, tokens=8191, cap=8191, adapters=3, rank=32, ends="4096,5120,6144", none=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "linear8", "lora"))
    if op == "norm":
        tokens = _log(rng, 1, 8191)
        bf16 = rng.random() < 0.5
        return dict(op=op, tokens=tokens, cap=tokens + rng.randint(0, 100), width=_log(rng, 40, min(16000, 8191 * 4096 // tokens)), normed=rng.random() < 0.75,
                    residual=rng.random() < 0.6, bf16=bf16, fp8=not bf16 or rng.random() < 0.6, pad=rng.choice((0, 0, 16, 48)))
    if op == "linear8":
        tokens = _log(rng, 1, 2176)
        gated = rng.random() < 0.3
        return dict(op=op, tokens=tokens, cap=tokens + rng.randint(0, 200), k=_log(rng, 17, 6000), n=_log(rng, 9, 6000 if gated else 12000),
                    act=rng.choice(ACTS), bias=rng.random() < 0.5, gated=gated, residual=rng.random() < 0.5)
    B = _log(rng, 1, 64)
    tokens = rng.randint(B, B * rng.choice((1, 4, 17, 17, 100)))
    gated = rng.random() < 0.25
    rank = rng.choice((8, 16, 16, 32, 64, 24))
    slices = 2 if gated else rng.choice((1, 1, 2, 3))
    sizes = [8 * _log(rng, 3, 700)] * 2 if gated else [_log(rng, 20, 4100) for _ in range(slices)]
    return dict(op=op, B=B, tokens=tokens, cap=tokens + rng.randint(0, 100), k=_log(rng, 40, 6000), adapters=_log(rng, 1, 40), rank=rank,
                ends=",".join(str(int(e)) for e in np.cumsum(sizes)), act=rng.choice(ACTS) if gated or rng.random() < 0.2 else "none", gated=gated,
                none=rng.random() < 0.7)


# ------------------------------------------------------------------------------------------- what follows from the case

def _ends(c):
    return [int(e) for e in c["ends"].split(",")]


def _adapters(c):
    """Adapter of each request, before they are shuffled: every eighth has none where the case says so."""
    return [-1 if c["none"] and i % 8 == 7 else i % c["adapters"] for i in range(c["B"])]


def work(c):
    t = c["tokens"]
    if c["op"] == "norm":
        per = 2 + (4 if c["residual"] else 0) + (2 if c["bf16"] else 0) + (1 if c["fp8"] else 0)
        return {"bytes": t * c["width"] * per + (4 * t if c["fp8"] else 0) + (2 * c["width"] if c["normed"] else 0), "flops": 8 * t * c["width"]}
    if c["op"] == "linear8":
        k, n, g = c["k"], c["n"], 2 if c["gated"] else 1
        return {"bytes": t * k + g * n * k + 2 * t * n * (2 if c["residual"] else 1) + 4 * t + 4 * g * n + (2 * g * n if c["bias"] else 0),
                "flops": 2 * g * t * n * k}
    ids, ends, r, k = _adapters(c), _ends(c), c["rank"], c["k"]
    used, live, n = len(set(ids) - {-1}), t * sum(i >= 0 for i in ids) // c["B"], ends[-1]
    return {"bytes": 2 * (live * k + used * r * (len(ends) * k + n) + t * n + t * (n // 2 if c["gated"] else n)),
            "flops": 2 * live * r * (len(ends) * k + n)}


# -------------------------------------------------------------------------------------------------------------- prepare

def _int(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _padded(gen, rows, cols, step, extra=0):
    """Rows that start on a multiple of `step` elements."""
    return _normal(gen, rows, -(-cols // step) * step + extra)[:, :cols]


def _fp8_rows(x):
    """8-bit rows (16 bytes aligned) with a scale each."""
    rows, cols = x.shape
    scale = x.float().abs().amax(1).clamp(min=LEAST) / E4M3_MAX
    y = torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.float8_e4m3fn, device="cuda")
    y[:, :cols] = (x.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return y[:, :cols], scale


def _context():
    """A serving process makes one context for its model and keeps it."""
    if "one" not in _contexts:
        from paper_2607_14647_b200 import binding
        _contexts["one"] = binding.Context(max_B=64, max_gamma=16, n_q_heads=32, n_kv_heads=8, head_dim=128, max_pages_per_req=1024)
    return _contexts["one"]


def prepare(c, seed):
    rng = np.random.default_rng([seed, 2])
    gen = torch.Generator("cuda").manual_seed(seed)
    s = {"norm": _prepare_norm, "linear8": _prepare_linear8, "lora": _prepare_lora}[c["op"]](c, rng, gen)
    if own:
        s["ctx"] = _context()
    return s


def _prepare_norm(c, rng, gen):
    T, cap, w = c["tokens"], c["cap"], c["width"]
    x = _padded(gen, cap, w, 8, c["pad"])
    stream = _padded(gen, cap, w, 8, c["pad"]) if c["residual"] else None
    if stream is not None:  # a residual stream: rows of different sizes, a few columns far above the others
        loud = torch.zeros(w, device="cuda")
        loud[torch.tensor(rng.permutation(w)[: max(1, w // 500)], device="cuda")] = 30.0
        stream.mul_((torch.exp(torch.randn((cap, 1), generator=gen, device="cuda")) * (1.0 + loud)).to(torch.bfloat16))
    return dict(c=c, T=T, x=x, stream=stream, cu=_int([0, T]), gain=(1 + 0.2 * _normal(gen, w)) if c["normed"] else None,
                h=torch.zeros((cap, w), dtype=torch.bfloat16, device="cuda") if c["residual"] else None,
                out=torch.zeros((cap, w), dtype=torch.bfloat16, device="cuda") if c["bf16"] else None,
                out8=torch.zeros((cap, -(-w // 16) * 16), dtype=torch.float8_e4m3fn, device="cuda")[:, :w] if c["fp8"] else None,
                scale8=torch.zeros(cap, dtype=torch.float32, device="cuda") if c["fp8"] else None)


def _prepare_linear8(c, rng, gen):
    k, n, cap = c["k"], c["n"], c["cap"]

    def weight():
        return _fp8_rows(_normal(gen, n, k) / math.sqrt(k))

    def bias():
        return _normal(gen, n) if c["bias"] else None

    a, a_scale = _fp8_rows(_normal(gen, cap, k))
    w, w_scale = weight()
    w2, w2_scale = weight() if c["gated"] else (None, None)
    return dict(c=c, T=c["tokens"], a=a, a_scale=a_scale, w=w, w_scale=w_scale, bias=bias(), w2=w2, w2_scale=w2_scale,
                bias2=bias() if c["gated"] else None, residual=_normal(gen, cap, n) if c["residual"] else None, cu=_int([0, c["tokens"]]),
                out=torch.zeros((cap, n), dtype=torch.bfloat16, device="cuda"))


def _prepare_lora(c, rng, gen):
    B, T, cap, k, r, m, ends = c["B"], c["tokens"], c["cap"], c["k"], c["rank"], c["adapters"], _ends(c)
    extra = np.bincount(rng.integers(0, B, T - B), minlength=B)  # every request one row at least
    n, sr, kp = ends[-1], len(ends) * r, -(-k // 8) * 8
    ids = rng.permutation(_adapters(c))
    return dict(c=c, T=T, x=_padded(gen, cap, k, 8), a=(_normal(gen, m, sr, kp) / math.sqrt(k))[:, :, :k], b=0.5 * _normal(gen, m, n, r),
                scale=0.5 + torch.rand(m, generator=gen, device="cuda"), ids=_int(ids), base=_normal(gen, cap, n), counts=_int(1 + extra),
                cu=_int(np.concatenate([[0], np.cumsum(1 + extra)])), ends=ends,
                out=torch.zeros((cap, n // 2 if c["gated"] else n), dtype=torch.bfloat16, device="cuda"))


# ------------------------------------------------------------------------------------------------------------------ run

def run(s):
    return {"norm": _run_norm, "linear8": _run_linear8, "lora": _run_lora}[s["c"]["op"]](s)


def _norm_outputs(s):
    return {k: s[k] for k in ("h", "out", "out8", "scale8") if s[k] is not None}


def _run_norm(s):
    c, T = s["c"], s["T"]
    if own:
        if c["normed"]:
            s["ctx"].rms_norm(s["x"], s["cu"], c["cap"], gain=s["gain"], rms_eps=EPS, residual=s["stream"], h_out=s["h"], out=s["out"], out8=s["out8"],
                              scale8=s["scale8"])
        else:
            s["ctx"].quantize(s["x"], s["cu"], c["cap"], residual=s["stream"], h_out=s["h"], out=s["out"], out8=s["out8"], scale8=s["scale8"])
        return _norm_outputs(s)
    y = s["x"][:T].float()
    if c["residual"]:
        y = y + s["stream"][:T].float()
        s["h"][:T] = y.to(torch.bfloat16)
    if c["normed"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * s["gain"].float()
    if c["bf16"]:
        s["out"][:T] = y.to(torch.bfloat16)
    if c["fp8"]:
        scale = y.abs().amax(1).clamp(min=LEAST) / E4M3_MAX
        s["out8"][:T] = (y / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        s["scale8"][:T] = scale
    return _norm_outputs(s)


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


def _run_linear8(s):
    c = s["c"]
    if own:
        s["ctx"].linear8(s["a"], s["a_scale"], s["w"], s["w_scale"], s["cu"], c["cap"], out=s["out"], bias=s["bias"], act=c["act"], w2=s["w2"],
                         w2_scale=s["w2_scale"], bias2=s["bias2"], residual=s["residual"])
        return s["out"]
    T = s["T"]
    a = s["a"][:T].float() * s["a_scale"][:T, None]

    def product(w, scale, bias):
        y = torch.matmul(a, (w.float() * scale[:, None]).t())
        return y if bias is None else y + bias.float()

    y = _activated(product(s["w"], s["w_scale"], s["bias"]), c["act"])
    if c["gated"]:
        y = y * product(s["w2"], s["w2_scale"], s["bias2"])
    if c["residual"]:
        y = y + s["residual"][:T].float()
    s["out"][:T] = y.to(torch.bfloat16)
    return s["out"]


def _run_lora(s):
    c = s["c"]
    if own:
        s["ctx"].lora(s["x"], s["a"], s["b"], s["ids"], s["base"], s["cu"], c["cap"], out=s["out"], scale=s["scale"], slices=s["ends"], act=c["act"],
                      gated=c["gated"])
        return s["out"]
    T, r, m, ends = s["T"], c["rank"], c["adapters"], s["ends"]
    n, sr = ends[-1], len(ends) * r
    ids = torch.repeat_interleave(s["ids"].long(), s["counts"].long(), output_size=T)
    mine = (ids[:, None] == torch.arange(m, device=ids.device)).float() * s["scale"]  # [T, adapters]
    low = torch.matmul(s["x"][:T].float(), s["a"].float().reshape(m * sr, c["k"]).t()).reshape(T, m, sr) * mine[:, :, None]
    b = s["b"].float()
    starts = [0] + ends[:-1]
    delta = torch.cat([torch.matmul(low[:, :, i * r:(i + 1) * r].reshape(T, m * r), b[:, lo:hi].transpose(1, 2).reshape(m * r, hi - lo))
                       for i, (lo, hi) in enumerate(zip(starts, ends))], 1)
    y = s["base"][:T].float() + delta
    y = _activated(y[:, :n // 2], c["act"]) * y[:, n // 2:] if c["gated"] else _activated(y, c["act"])
    s["out"][:T] = y.to(torch.bfloat16)
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------- exact

def _exact_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":  # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def exact(c, seed):
    """The operators' definitions in 64 bits, a block of rows or an adapter at a time; 8-bit values before their rounding."""
    s, T = prepare(c, seed), c["tokens"]
    if c["op"] == "norm":
        outs = {k: v.double() for k, v in _norm_outputs(s).items()}
        for i in range(0, T, 512):
            rows = slice(i, min(T, i + 512))
            h = s["x"][rows].double()
            if c["residual"]:
                h += s["stream"][rows].double()
                outs["h"][rows] = h
            if c["normed"]:
                h = s["gain"].double() * h / (h.pow(2).sum(1, keepdim=True) / c["width"] + EPS).sqrt()
            if c["bf16"]:
                outs["out"][rows] = h
            if c["fp8"]:
                top = torch.maximum(h.max(1).values, -h.min(1).values).clamp(min=LEAST)
                outs["scale8"][rows] = top / E4M3_MAX
                outs["out8"][rows] = h * (E4M3_MAX / top)[:, None]
        return outs
    if c["op"] == "linear8":
        y = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for i in range(0, T, 512):
            rows = slice(i, min(T, i + 512))
            x = s["a"][rows].double()

            def product(w, scale, bias):
                z = torch.einsum("tk,nk->tn", x, w.double()) * s["a_scale"][rows].double()[:, None] * scale.double()
                return z if bias is None else z + bias.double()

            z = _exact_act(product(s["w"], s["w_scale"], s["bias"]), c["act"])
            if c["gated"]:
                z = z * product(s["w2"], s["w2_scale"], s["bias2"])
            y[rows] = z if s["residual"] is None else z + s["residual"][rows].double()
        return y
    y = torch.zeros(s["base"].shape, dtype=torch.float64, device="cuda")
    cu, ids, r = s["cu"].tolist(), s["ids"].tolist(), c["rank"]
    for i in range(c["B"]):
        rows = slice(cu[i], cu[i + 1])
        y[rows] = s["base"][rows].double()
        if ids[i] >= 0:
            lo = 0
            for j, hi in enumerate(s["ends"]):
                down = s["a"][ids[i], j * r:(j + 1) * r].double()
                y[rows, lo:hi] += float(s["scale"][ids[i]]) * ((s["x"][rows].double() @ down.T) @ s["b"][ids[i], lo:hi].double().T)
                lo = hi
    half = s["ends"][-1] // 2
    z = _exact_act(y[:, :half], c["act"]) * y[:, half:] if c["gated"] else _exact_act(y, c["act"])
    z[T:] = 0.0
    return z
