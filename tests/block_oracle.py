"""The gated delta rule, layer norm and dropout from their definitions, in 64 bits on the CPU."""
import math

import torch

U_BF16 = 2.0 ** -8     # unit roundoff of bfloat16
U_F32 = 2.0 ** -24


def f64(t):
    return None if t is None else t.detach().cpu().double()


def delta(q, k, v, log_decay, beta, state=None, lengths=None, scale=1.0):
    """(out [B, L, H, dv], last state [B, H, dk, dv]), token by token; inputs in 64 bits keep their graph."""
    B, L, H = log_decay.shape
    dk, dv = q.shape[3], v.shape[3]
    heads = lambda t: t.repeat_interleave(H // t.shape[2], 2)  # noqa: E731
    q, k, v = heads(q), heads(k), heads(v)
    S = torch.zeros(B, H, dk, dv, dtype=torch.float64) if state is None else state
    n = torch.full((B,), L) if lengths is None else lengths.cpu().long().clamp(0, L)
    out = []
    for t in range(L):
        here = (t < n)[:, None, None, None]
        D = S * torch.exp(log_decay[:, t])[..., None, None]
        u = beta[:, t, :, None] * (v[:, t] - (k[:, t, :, None] @ D)[..., 0, :])
        S = torch.where(here, D + k[:, t, ..., None] * u[..., None, :], S)
        o = scale * (q[:, t, :, None] @ S)[..., 0, :]
        out.append(torch.where(here[..., 0], o, torch.zeros_like(o)))
    return torch.stack(out, 1) if L else torch.zeros(B, 0, H, dv, dtype=torch.float64), S


def cleared(t, lengths):
    """[B, L, ...] in 64 bits with zeros behind the lengths (nothing there may be read)."""
    t = f64(t)
    if lengths is None:
        return t
    here = torch.arange(t.shape[1]) < lengths.cpu()[:, None]
    return torch.where(here.reshape(here.shape + (1,) * (t.dim() - 2)), t, torch.zeros_like(t))


def delta_of(q, k, v, log_decay, beta, state=None, lengths=None, scale=1.0):
    return delta(*(cleared(t, lengths) for t in (q, k, v, log_decay, beta)), f64(state), lengths, scale)


def delta_backward(dout, q, k, v, log_decay, beta, state=None, dstate=None, lengths=None, scale=1.0):
    """(dq, dk, dv, dlog_decay, dbeta, gradient of the state)"""
    B, _, H = log_decay.shape
    state = torch.zeros(B, H, q.shape[3], v.shape[3], dtype=torch.float64) if state is None else f64(state)
    leaves = [cleared(t, lengths) for t in (q, k, v, log_decay, beta)] + [state]
    leaves = [t.clone().requires_grad_() for t in leaves]
    out, last = delta(*leaves, lengths, scale)
    last_grad = torch.zeros_like(last) if dstate is None else f64(dstate)
    grads = torch.autograd.grad((out, last), leaves, (cleared(dout, lengths), last_grad), allow_unused=True)
    return [torch.zeros_like(x) if g is None else g for g, x in zip(grads, leaves)]


def delta_decay_sizes(dout, q, k, v, log_decay, beta, state, dstate, lengths=None, scale=1.0):
    """|D_t| |E_t| [B, L, H]: of the decayed state that a token sees and of its gradient, whose product the gradient of the decay's logarithm is."""
    B, L, H = log_decay.shape
    dout, q, k, v, log_decay, beta = (cleared(t, lengths) for t in (dout, q, k, v, log_decay, beta))
    q, k, v = (t.repeat_interleave(H // t.shape[2], 2) for t in (q, k, v))
    n = torch.full((B,), L) if lengths is None else lengths.cpu().long().clamp(0, L)
    S, R, seen = f64(state), f64(dstate), []
    for t in range(L):
        D = S * torch.exp(log_decay[:, t])[..., None, None]
        u = beta[:, t, :, None] * (v[:, t] - (k[:, t, :, None] @ D)[..., 0, :])
        S = torch.where((t < n)[:, None, None, None], D + k[:, t, ..., None] * u[..., None, :], S)
        seen.append(D.flatten(2).norm(dim=-1))
    sizes = [None] * L
    for t in range(L - 1, -1, -1):
        here = (t < n)[:, None, None, None]
        E = R + scale * q[:, t, ..., None] * dout[:, t, :, None]
        E = E - k[:, t, ..., None] * (beta[:, t, :, None] * (k[:, t, :, None] @ E)[..., 0, :])[..., None, :]
        sizes[t] = seen[t] * E.flatten(2).norm(dim=-1) * here[..., 0, 0]
        R = torch.where(here, E * torch.exp(log_decay[:, t])[..., None, None], R)
    return torch.stack(sizes, 1)


def norm(x, weight, bias, eps):
    x = f64(x)
    y = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + eps)
    y = y if weight is None else y * f64(weight)
    return y if bias is None else y + f64(bias)


def norm_backward(dout, x, weight, eps):
    leaf = f64(x).requires_grad_()
    w = (torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else f64(weight)).requires_grad_()
    b = torch.zeros(x.shape[-1], dtype=torch.float64, requires_grad=True)
    y = (leaf - leaf.mean(-1, keepdim=True)) / torch.sqrt(leaf.var(-1, unbiased=False, keepdim=True) + eps)
    return torch.autograd.grad(y * w + b, (leaf, w, b), f64(dout))


def philox(counter, key):
    """Philox4x32-10 of one counter (four words) and key (two)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(n, p, seed, offset, first=0):
    """Which of the elements first .. first + n stay."""
    border, words = min(65535, math.floor(p * 65536 + 0.5)), {}
    keep = []
    for i in range(first, first + n):
        block = i // 8
        if block not in words:
            words[block] = philox((block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        keep.append((words[block][i % 8 // 2] >> (16 * (i & 1)) & 0xFFFF) >= border)
    return torch.tensor(keep)
