"""Plain 64-bit forms of the attention-block operators (rotary append, shared-prefix attention, linear), for the tests."""
import numpy as np


def bf16_values(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def rope_rows(x, pos, inv_freq, interleaved, gain=None, eps=0.0):
    """x fp64 [T, H, D] at positions pos: optional RMS norm per head, then the rotation of the first 2 len(inv_freq) elements."""
    x = np.array(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    R = 2 * len(inv_freq)
    angle = np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
    c, s = np.cos(angle), np.sin(angle)
    a, b = (np.arange(0, R, 2), np.arange(1, R, 2)) if interleaved else (np.arange(R // 2), np.arange(R // 2, R))
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def prefix_len_of(req, cu_group, prefix_lens):
    return int(prefix_lens[np.searchsorted(np.asarray(cu_group), req, side="right") - 1])


def prefix_attn(q, k_cache, v_cache, block_table, ctx_lens, cu_q, cu_group, prefix_lens, prefix_table, scale):
    """out fp64 [T, Hq, D], lse [T, Hq]: softmax over the group's shared positions and the request's own ones; also the
    weighted mean of |v| (what relative errors of the weights act on) and the largest sum_c |q_c k_c| of a row's scores."""
    T, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    out, lse, mean_abs, abs_score = np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    G = np.asarray(cu_group)
    for i in range(len(ctx_lens)):
        g = int(np.searchsorted(G, i, side="right") - 1)
        P, n = int(prefix_lens[g]), int(cu_q[i + 1] - cu_q[i])
        total = int(ctx_lens[i]) + n
        rows = [(prefix_table[g, j // 16], j % 16) if j < P else (block_table[i, (j - P) // 16], (j - P) % 16) for j in range(total)]
        page, slot = np.array([r[0] for r in rows]), np.array([r[1] for r in rows])
        k, v = k_cache[page, :, slot], v_cache[page, :, slot]                  # [total, Hkv, D]
        for h in range(Hq):
            s = q[cu_q[i]:cu_q[i + 1], h] @ k[:, h // (Hq // Hkv)].T * scale   # [n, total]
            s[np.arange(total)[None, :] > int(ctx_lens[i]) + np.arange(n)[:, None]] = -np.inf
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            out[cu_q[i]:cu_q[i + 1], h] = np.where(p > 0, p, 0) @ v[:, h // (Hq // Hkv)] / p.sum(1, keepdims=True)
            lse[cu_q[i]:cu_q[i + 1], h] = (m + np.log(p.sum(1, keepdims=True)))[:, 0]
            mean_abs[cu_q[i]:cu_q[i + 1], h] = p @ np.abs(v[:, h // (Hq // Hkv)]) / p.sum(1, keepdims=True)
            abs_score[cu_q[i]:cu_q[i + 1], h] = (np.abs(q[cu_q[i]:cu_q[i + 1], h]) @ np.abs(k[:, h // (Hq // Hkv)]).T * scale).max(1)
    return out, lse, mean_abs, abs_score


def linear(a, w, bias=None, act="none", w2=None, bias2=None, residual=None):
    import math
    z = a @ w.T + (0 if bias is None else bias)
    if act == "relu":
        z = np.maximum(z, 0)
    elif act == "gelu":
        z = 0.5 * z * np.vectorize(math.erfc)(-z / math.sqrt(2))               # (1 + erf cancels far below zero)
    elif act == "gelu_tanh":
        with np.errstate(over="ignore"):                                       # (1 + tanh u) / 2 = 1 / (1 + e^-2u)
            z = z / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    elif act == "silu":
        with np.errstate(over="ignore"):
            z = z / (1 + np.exp(-z))
    if w2 is not None:
        z = z * (a @ w2.T + (0 if bias2 is None else bias2))
    return z if residual is None else z + residual


def rms_norm(x, residual, normed, gain, eps, plus_one):
    """(h, y) of dcut_rms_norm in 64 bits."""
    h = x if residual is None else x + residual
    y = h
    if normed:
        big = np.maximum(np.abs(h).max(1, keepdims=True), 1.0)                 # (squares of large values)
        y = h / big / np.sqrt(((h / big) ** 2).mean(1, keepdims=True) + eps / big / big)
        if gain is not None:
            y = y * (gain + (1.0 if plus_one else 0.0))
    return h, y
