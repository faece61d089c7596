"""The operators of a decoder layer behind shared prefixes, one after the other as a server runs them: QKV projection with
bias, query/key norm and rotation with the append to the cache, attention over shared and own pages, output projection onto
the residual stream, gated MLP.  A first step appends each request's own context, a second verifies drafts on it; own pages
start as NaN.  Each operator's output is checked against its formula in 64 bits on the operands it was given (tolerances:
the operators' own tests)."""
import numpy as np
import pytest
import torch

from tests import test_gpu_linear as lin
from tests import test_gpu_prefix_attn as attn
from tests.plain_reference import bf16_values, rope_rows
from tests.test_gpu_rope_append import _near

pytestmark = pytest.mark.gpu


def _i32(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self, hq, hkv, d, hidden, inner, interleaved):
        from paper_2607_14647_b200 import binding
        self.hq, self.hkv, self.d, self.hidden, self.inner, self.interleaved = hq, hkv, d, hidden, inner, interleaved
        self.sizes, self.plens = np.array([3, 2, 4]), np.array([197, 0, 64])
        self.own, self.draft = np.array([30, 1, 17, 36, 16, 3, 9, 33, 32]), np.array([1, 9, 17, 3, 1, 16, 17, 2, 5])
        B, G = len(self.own), len(self.sizes)
        self.pre = np.repeat(self.plens, self.sizes)
        rng = np.random.default_rng(d)
        own_pages, shared = -(-(self.own + self.draft) // 16), -(-self.plens // 16)
        pool = int(own_pages.sum() + shared.sum())
        ids = rng.permutation(pool)
        self.table, self.ptable, at = np.full((B, own_pages.max()), -1), np.full((G, max(1, shared.max())), -1), 0
        for rows, need in ((self.table, own_pages), (self.ptable, shared)):
            for i, n in enumerate(need):
                rows[i, :n] = ids[at:at + n]
                at += n
        g = torch.Generator("cuda").manual_seed(d)
        self.n = lambda *s, scale=1.0: (scale * torch.randn(s, generator=g, device="cuda")).to(torch.bfloat16)
        self.kc, self.vc = (torch.full((pool, hkv, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv")
        for i, p in enumerate(self.plens):
            for j in range(-(-p // 16)):
                rows = min(16, p - 16 * j)
                self.kc[self.ptable[i, j], :, :rows], self.vc[self.ptable[i, j], :, :rows] = self.n(hkv, rows, d), self.n(hkv, rows, d)
        n_qkv, h = (hq + 2 * hkv) * d, hidden ** -0.5
        self.w_qkv, self.b_qkv, self.w_o, self.b_o = self.n(n_qkv, hidden, scale=h), self.n(n_qkv), self.n(hidden, hq * d, scale=(hq * d) ** -0.5), self.n(hidden)
        self.w_g, self.w_u, self.w_d = self.n(inner, hidden, scale=h), self.n(inner, hidden, scale=h), self.n(hidden, inner, scale=inner ** -0.5)
        self.q_gain, self.k_gain = 1 + 0.2 * self.n(d), 1 + 0.2 * self.n(d)
        self.freq = binding.rope_inv_freq(1e4, d)
        self.groups = binding.PrefixGroups(_i32(np.concatenate([[0], np.cumsum(self.sizes)])), _i32(self.plens), _i32(self.ptable))
        self.d_table = _i32(self.table)
        self.ctx = binding.Context(max_B=B, max_gamma=35, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_pages_per_req=32)
        self.ctx.enable_prefix_attn(G)

    def step(self, counts, ctx_own, pad):
        """What one step of the loop feeds the operators: `counts` rows per request on top of `ctx_own` own positions."""
        req = np.repeat(np.arange(len(counts)), counts)
        cu = np.concatenate([[0], np.cumsum(counts)])
        T, cap = len(req), len(req) + pad
        pos = (self.pre + ctx_own)[req] + np.arange(T) - cu[req]
        fill = lambda x: np.concatenate([x, np.full(pad, -1)])
        x = self.n(cap, self.hidden)
        x[T:] = float("nan")
        return dict(T=T, cap=cap, host=(req, pos, cu, counts, ctx_own), x=x, req=_i32(fill(req)), pos=_i32(fill(pos)), cu=_i32(cu), ctx=_i32(self.pre + ctx_own))

    def run(self, s):
        c, cap, cu = self.ctx, s["cap"], s["cu"]
        r = dict(qkv=c.linear(s["x"], self.w_qkv, cu, cap, bias=self.b_qkv))
        qkv = r["qkv"].view(cap, self.hq + 2 * self.hkv, self.d)
        r["q"] = c.rope_append(qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:], self.freq, self.kc, self.vc,
                               self.d_table, s["req"], s["pos"], cap, cu_q=cu, interleaved=self.interleaved, q_gain=self.q_gain, k_gain=self.k_gain,
                               groups=self.groups)
        r["attn"] = torch.full((cap, self.hq, self.d), 7.0, dtype=torch.bfloat16, device="cuda")
        c.prefix_attn(r["q"], self.kc, self.vc, self.d_table, s["ctx"], cu, cap, self.groups, out=r["attn"])
        r["mid"] = c.linear(r["attn"].view(cap, -1), self.w_o, cu, cap, bias=self.b_o, residual=s["x"])
        r["act"] = c.linear(r["mid"], self.w_g, cu, cap, act="silu", w2=self.w_u)
        r["y"] = c.linear(r["act"], self.w_d, cu, cap, residual=r["mid"])
        return r

    def check(self, s, r):
        T, (req, pos, cu, counts, ctx_own) = s["T"], s["host"]
        case = lambda a, w, **kw: dict(dict(a=a, w=w, T=T, bias=None, w2=None, bias2=None, residual=None), **kw)
        lin.check(case(s["x"], self.w_qkv, bias=self.b_qkv), r["qkv"])
        qkv = bf16_values(r["qkv"])[:T].reshape(T, -1, self.d)
        freq, page = self.freq.cpu().numpy(), self.table[req, (pos - self.pre[req]) // 16]
        at = (pos - self.pre[req]) % 16
        want_q = rope_rows(qkv[:, :self.hq], pos, freq, self.interleaved, bf16_values(self.q_gain), 1e-6)
        want_k = rope_rows(qkv[:, self.hq:self.hq + self.hkv], pos, freq, self.interleaved, bf16_values(self.k_gain), 1e-6)
        kc, vc = bf16_values(self.kc), bf16_values(self.vc)
        assert _near(bf16_values(r["q"])[:T], want_q, want_q) and _near(kc[page, :, at], want_k, want_k)
        assert np.array_equal(vc[page, :, at], qkv[:, self.hq + self.hkv:])
        a = dict(T=T, d=self.d, q=r["q"][:T], kc_plain=np.nan_to_num(kc), vc_plain=np.nan_to_num(vc), table=self.table, ctx=self.pre + ctx_own, cu=cu,
                 cu_group=np.concatenate([[0], np.cumsum(self.sizes)]), plens=self.plens, ptable=self.ptable)
        attn.check(a, r["attn"], None)
        assert bool((r["attn"][T:] == 7).all())
        lin.check(case(r["attn"].view(s["cap"], -1), self.w_o, bias=self.b_o, residual=s["x"]), r["mid"])
        lin.check(case(r["mid"], self.w_g, w2=self.w_u), r["act"], "silu")
        lin.check(case(r["act"], self.w_d, residual=r["mid"]), r["y"])


@pytest.mark.parametrize("hq,hkv,d,interleaved", [(8, 2, 128, False), (4, 4, 64, True)])
def test_a_layer_step_by_step_and_captured(hq, hkv, d, interleaved):
    layer = Layer(hq, hkv, d, 320, 776, interleaved)
    zeros = np.zeros_like(layer.own)
    first = layer.step(layer.own, zeros, 0)
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
        for t in r.values():
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert layer.ctx.poll_device_status() == 0
        for name in r:
            assert torch.equal(r[name][:second["T"]], eager[name][:second["T"]]), name
    assert torch.equal(layer.kc.view(torch.int16), kc.view(torch.int16)) and torch.equal(layer.vc.view(torch.int16), vc.view(torch.int16))
