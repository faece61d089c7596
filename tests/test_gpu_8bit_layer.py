"""The operators of a decoder layer of a target held in 8 bits whose requests carry adapters, one after the other as a server runs them: norm to
8 bits, shared projection, adapters, rotation with the append to the cache, attention, and so on to the residual stream behind the MLP.  A
first step appends each request's context, a second verifies drafts on it.  Each operator's output is checked against its formula in 64 bits
on the operands it was given (tolerances: the operators' own tests)."""
import numpy as np
import pytest
import torch

from tests import test_gpu_linear8 as lin8
from tests import test_gpu_lora as adapters
from tests import test_gpu_rms_norm as norm
from tests.gpu_helpers import attn_tolerance_ok
from tests.plain_reference import bf16_values, prefix_attn, rope_rows
from tests.test_gpu_rope_append import _near

pytestmark = pytest.mark.gpu


def _i32(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self, hq, hkv, d, hidden, inner, rank, ids):
        from paper_2607_14647_b200 import binding
        self.b, self.hq, self.hkv, self.d, self.hidden, self.inner, self.ids = binding, hq, hkv, d, hidden, inner, np.array(ids)
        self.own, self.draft = np.array([30, 1, 17, 36, 16, 3]), np.array([1, 9, 17, 3, 17, 5])
        B, m = len(self.own), max(ids) + 1
        pages = -(-(self.own + self.draft) // 16)
        perm, at = np.random.default_rng(d).permutation(int(pages.sum())), 0
        self.table = np.full((B, pages.max()), -1)
        for i, n in enumerate(pages):
            self.table[i, :n] = perm[at:at + n]
            at += n
        g = torch.Generator("cuda").manual_seed(d + rank)
        self.n = lambda *s, scale=1.0: (scale * torch.randn(s, generator=g, device="cuda")).to(torch.bfloat16)
        self.kc, self.vc = (torch.full((int(pages.sum()), hkv, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv")
        self.ctx = binding.Context(max_B=B, max_gamma=35, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_pages_per_req=32)
        n_q, n_kv = hq * d, hkv * d
        self.ends = dict(qkv=[n_q, n_q + n_kv, n_q + 2 * n_kv], o=[hidden], gu=[inner, 2 * inner], down=[hidden])
        self.k = dict(qkv=hidden, o=n_q, gu=hidden, down=inner)
        self.w, self.a, self.bb = {}, {}, {}
        for name, ends in self.ends.items():
            k = self.k[name]
            self.w[name] = self.ctx.quantize(self.n(ends[-1], k, scale=k ** -0.5), None, ends[-1])       # rows of a weight: its output channels
            self.a[name], self.bb[name] = self.n(m, len(ends) * rank, k, scale=k ** -0.5), self.n(m, ends[-1], rank, scale=0.3)
        self.scale = 0.5 + torch.rand(m, generator=g, device="cuda")
        self.gain, self.gain2 = 1 + 0.2 * self.n(hidden), 1 + 0.2 * self.n(hidden)
        self.freq, self.adapter, self.d_table = binding.rope_inv_freq(1e4, d), _i32(self.ids), _i32(self.table)

    def step(self, counts, ctx_own, pad):
        req = np.repeat(np.arange(len(counts)), counts)
        cu = np.concatenate([[0], np.cumsum(counts)])
        T, cap = len(req), len(req) + pad
        pos = ctx_own[req] + np.arange(T) - cu[req]
        fill = lambda x: np.concatenate([x, np.full(pad, -1)])
        x = self.n(cap, self.hidden)
        x[T:] = float("nan")
        return dict(T=T, cap=cap, host=(req, pos, cu, ctx_own), x=x, req=_i32(fill(req)), pos=_i32(fill(pos)), cu=_i32(cu), ctx=_i32(ctx_own))

    def run(self, s):
        c, cap, cu, r, b = self.ctx, s["cap"], s["cu"], {}, self.b
        bf = lambda w: torch.empty((cap, w), dtype=torch.bfloat16, device="cuda")

        def project(name, x8, x, residual=None, **kw):
            r[name + "_base"] = c.linear8(x8[0], x8[1], *self.w[name], cu, cap, residual=residual)
            r[name] = c.lora(x, self.a[name], self.bb[name], self.adapter, r[name + "_base"], cu, cap, scale=self.scale, slices=self.ends[name], **kw)
            return r[name]

        r["n"], r["n8"] = bf(self.hidden), (b.rows8(cap, self.hidden), torch.empty(cap, device="cuda"))
        c.rms_norm(s["x"], cu, cap, gain=self.gain, out=r["n"], out8=r["n8"][0], scale8=r["n8"][1])
        qkv = project("qkv", r["n8"], r["n"]).view(cap, self.hq + 2 * self.hkv, self.d)
        r["q"] = c.rope_append(qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:], self.freq, self.kc, self.vc, self.d_table,
                               s["req"], s["pos"], cap, cu_q=cu)
        r["attn"] = c.verify_attn(r["q"], self.kc, self.vc, self.d_table, s["ctx"], cu, cap).view(cap, -1)
        r["attn8"] = c.quantize(r["attn"], cu, cap)
        o = project("o", r["attn8"], r["attn"])
        r["h"], r["n2"], r["n28"] = bf(self.hidden), bf(self.hidden), (b.rows8(cap, self.hidden), torch.empty(cap, device="cuda"))
        c.rms_norm(o, cu, cap, gain=self.gain2, residual=s["x"], h_out=r["h"], out=r["n2"], out8=r["n28"][0], scale8=r["n28"][1])
        act = project("gu", r["n28"], r["n2"], act="silu", gated=True)
        r["act8"] = c.quantize(act, cu, cap)
        project("down", r["act8"], act, residual=r["h"])
        return r

    def check(self, s, r):
        T, (req, pos, cu, ctx_own) = s["T"], s["host"]

        def projected(name, x8, x, residual=None, act="none", gated=False):
            w, ws = self.w[name]
            lin8.check(dict(a=x8[0], a_scale=x8[1], w=w, w_scale=ws, w2=None, w2_scale=None, bias=None, bias2=None, residual=residual, T=T), r[name + "_base"])
            adapters.check(dict(x=x, a=self.a[name], b=self.bb[name], base=r[name + "_base"], ids=self.ids, hcu=cu, scale=self.scale, ends=self.ends[name],
                                gated=gated, width=r[name].shape[1]), r[name], act, untouched=False)

        def normed(x, o, normed=True, **kw):
            norm.check({k: o.get(k) for k in "hb8"}, dict(s=o["s"][:T]), x, T, normed, **kw)

        normed(s["x"], {"b": r["n"], "8": r["n8"][0], "s": r["n8"][1]}, gain=self.gain)
        projected("qkv", r["n8"], r["n"])
        qkv, freq = bf16_values(r["qkv"])[:T].reshape(T, -1, self.d), self.freq.cpu().numpy()
        page, at = self.table[req, pos // 16], pos % 16
        want_q, want_k = (rope_rows(v, pos, freq, False) for v in (qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv]))
        kc, vc = bf16_values(self.kc), bf16_values(self.vc)
        assert _near(bf16_values(r["q"])[:T], want_q, want_q) and _near(kc[page, :, at], want_k, want_k)
        assert np.array_equal(vc[page, :, at], qkv[:, self.hq + self.hkv:])
        B = len(ctx_own)
        want = prefix_attn(bf16_values(r["q"])[:T], np.nan_to_num(kc), np.nan_to_num(vc), self.table, ctx_own, cu, np.array([0, B]), np.array([0]),
                           np.zeros((1, 1), int), self.d ** -0.5)[0]
        ok, worst = attn_tolerance_ok(bf16_values(r["attn"])[:T].reshape(want.shape), want)
        assert ok, worst
        normed(r["attn"], {"8": r["attn8"][0], "s": r["attn8"][1]}, normed=False)
        projected("o", r["attn8"], r["attn"])
        normed(r["o"], {"h": r["h"], "b": r["n2"], "8": r["n28"][0], "s": r["n28"][1]}, gain=self.gain2, residual=s["x"])
        projected("gu", r["n28"], r["n2"], act="silu", gated=True)
        normed(r["gu"], {"8": r["act8"][0], "s": r["act8"][1]}, normed=False)
        projected("down", r["act8"], r["gu"], residual=r["h"])


def flat(r):
    for name, v in sorted(r.items()):
        for i, t in enumerate(v if isinstance(v, tuple) else (v,)):
            yield f"{name}{i}", t


@pytest.mark.parametrize("hq,hkv,d,rank,ids", [(8, 2, 128, 16, [0, 1, -1, 0, 2, 1]), (4, 4, 64, 40, [-1, 3, 3, 0, 2, -1])])
def test_a_layer_step_by_step_and_captured(hq, hkv, d, rank, ids):
    layer = Layer(hq, hkv, d, 328, 776, rank, ids)
    first = layer.step(layer.own, np.zeros_like(layer.own), 0)
    layer.check(first, layer.run(first))
    second = layer.step(layer.draft, layer.own, 5)
    eager = layer.run(second)
    assert layer.ctx.poll_device_status() == 0
    layer.check(second, eager)
    kc, vc = layer.kc.clone(), layer.vc.clone()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        r = layer.run(second)
    for _ in range(2):
        for _, t in flat(r):
            t.view(torch.uint8).zero_() if t.is_contiguous() else t.copy_(torch.zeros_like(t))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert layer.ctx.poll_device_status() == 0
        for (name, t), (_, e) in zip(flat(r), flat(eager)):
            assert torch.equal(t[:second["T"]].float(), e[:second["T"]].float()), name
    assert torch.equal(layer.kc.view(torch.int16), kc.view(torch.int16)) and torch.equal(layer.vc.view(torch.int16), vc.view(torch.int16))
