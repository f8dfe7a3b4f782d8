"""The sequence operators from their definitions, token by token in 64 bits on the CPU."""
import math

import torch

U_BF16 = 2.0 ** -8     # unit roundoff of bfloat16
U_F32 = 2.0 ** -24


def f64(t):
    return None if t is None else t.detach().cpu().double()


def attention(q, k, v, log_decay, state=None, lengths=None, scale=1.0):
    """(out [B, L, H, dv], last state [B, H, dk, dv])"""
    q, k, v, g, state = map(f64, (q, k, v, log_decay, state))
    B, L, H, dk = q.shape
    G, dv = v.shape[2:]
    S = torch.zeros(B, H, dk, dv, dtype=torch.float64) if state is None else state.clone()
    out = torch.zeros(B, L, H, dv, dtype=torch.float64)
    for b in range(B):
        n = L if lengths is None else max(0, min(L, int(lengths[b])))
        for h in range(H):
            lam, kv = math.exp(g[h]), h // (H // G)
            for t in range(n):
                S[b, h] = lam * S[b, h] + torch.outer(k[b, t, kv], v[b, t, kv])
                out[b, t, h] = scale * (q[b, t, h] @ S[b, h])
    return out, S


def attention_backward(dout, q, k, v, log_decay, state=None, dstate=None, lengths=None, scale=1.0):
    """(dq, dk, dv, gradient of state)"""
    dout, q, k, v, g, state, dstate = map(f64, (dout, q, k, v, log_decay, state, dstate))
    B, L, H, dk = q.shape
    G, dv = v.shape[2:]
    R0 = torch.zeros(B, H, dk, dv, dtype=torch.float64) if dstate is None else dstate.clone()
    dq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(B):
        n = L if lengths is None else max(0, min(L, int(lengths[b])))
        for h in range(H):
            lam, kv = math.exp(g[h]), h // (H // G)
            S = torch.zeros(dk, dv, dtype=torch.float64) if state is None else state[b, h].clone()
            for t in range(n):
                S = lam * S + torch.outer(k[b, t, kv], v[b, t, kv])
                dq[b, t, h] = scale * (S @ dout[b, t, h])
            R = R0[b, h]
            for t in range(n - 1, -1, -1):
                R = R + scale * torch.outer(q[b, t, h], dout[b, t, h])
                gk[b, t, kv] += R @ v[b, t, kv]
                gv[b, t, kv] += k[b, t, kv] @ R
                R = lam * R
            R0[b, h] = R
    return dq, gk, gv, R0


def turned(x, positions, freqs, layout, magnitude, inverse=False):
    x = f64(x).clone()
    B, L, H, D = x.shape
    n = len(freqs)
    for b in range(B):
        for t in range(L):
            p = t if positions is None else int(positions[b, t])
            for i in range(n):
                a = p * float(freqs[i])
                c, s = magnitude * math.cos(a), magnitude * math.sin(a)
                s = -s if inverse else s
                i0, i1 = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
                u, w = x[b, t, :, i0].clone(), x[b, t, :, i1].clone()
                x[b, t, :, i0], x[b, t, :, i1] = u * c - w * s, u * s + w * c
    return x


def normed(x, weight, eps):
    x = f64(x)
    y = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    return y if weight is None else y * f64(weight)


def norm_rotate(x, weight, positions, freqs, eps, layout, magnitude):
    return turned(normed(x, weight, eps), positions, freqs, layout, magnitude)


def norm_rotate_backward(dout, x, weight, positions, freqs, eps, layout, magnitude):
    """(dx, dweight)"""
    dy = turned(dout, positions, freqs, layout, magnitude, inverse=True)
    x = f64(x)
    D = x.shape[-1]
    root = (x.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    h = dy if weight is None else dy * f64(weight)
    dx = h / root - x * (h * x).sum(-1, keepdim=True) / (D * root ** 3)
    return dx, (dy * x / root).sum((0, 1, 2))
