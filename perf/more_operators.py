"""Timed work of the operators of a residual block over sequences: its norm, its memory and its dropout.

A learner of replayed sequences trains blocks x + dropout(memory(norm(x))), the actors beside it advance the memory by one token.

A *case* is a dict of plain values.  ``prepare`` makes what such a program has in hand, ``run`` is one pass through one
operator, ``work`` the bytes and operations that pass cannot do without, ``exact`` its outputs from the definition in
64 bits.  ``own`` says whether ``run`` takes the framework's operators or the plain form written here.

Forms (``"form"``):
  step    the gated delta rule, one token of many actors: the states are updated in place
  delta   the same over sequences (ragged where ``ragged``), from given states: outputs and final states
  train   its gradient: of queries, keys, values, decays, strengths and initial states
  norm    layer norm of rows
  grad    its gradient: of rows, weight and bias
  drop    dropout from a counter-based generator, added to a residual where ``residual`` (without one it is also the gradient)
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # 64 actors stepping together, a small recurrent policy: nothing but latency.
        dict(name="delta_actors", form="step", type="bf16", B=64, H=4, Q=4, K=4, V=4, dk=64, dv=64),
        # A fleet of 512 environments with a large policy: half a gigabyte of states read and written for one token each.
        dict(name="delta_fleet", form="step", type="bf16", B=512, H=16, Q=8, K=8, V=16, dk=128, dv=128),
        # A learner's batch of replayed stretches of up to 80 steps, each from its stored state, some cut short by an episode's end.
        dict(name="delta_replay", form="delta", type="bf16", B=64, L=80, H=4, Q=4, K=4, V=4, dk=64, dv=64, ragged=True),
        # Nothing here is a power of two: single precision, heads that share keys and values.
        dict(name="delta_odd", form="delta", type="f32", B=3, L=1001, H=6, Q=6, K=2, V=2, dk=48, dv=80, ragged=True),
        # One whole history of 65536 steps through a large policy, heads in pairs that share queries and keys: few rows, a long axis.
        dict(name="delta_long", form="delta", type="bf16", B=1, L=65536, H=16, Q=8, K=8, V=16, dk=128, dv=128, ragged=False),
        # The gradient for a batch of 32 replayed stretches of up to 512 steps; eight heads share two of keys and values.
        dict(name="delta_train_replay", form="train", type="bf16", B=32, L=512, H=8, Q=8, K=2, V=2, dk=64, dv=64, ragged=True),
        # The gradient through two long histories.
        dict(name="delta_train_long", form="train", type="bf16", B=2, L=8192, H=16, Q=16, K=16, V=16, dk=128, dv=128, ragged=False),
        # The hidden rows of 64 actors.
        dict(name="norm_actors", form="norm", type="f32", B=64, L=1, D=256),
        # The hidden rows of a learner's batch: 16 stretches of 2048 steps, 2048 wide.
        dict(name="norm_rows", form="norm", type="bf16", B=16, L=2048, D=2048),
        # Their gradient, on stretches and rows of odd sizes.
        dict(name="norm_grad_odd", form="grad", type="bf16", B=8, L=1023, D=1537),
        # What a block of that learner adds to its residual.
        dict(name="drop_rows", form="drop", type="bf16", B=16, L=2048, D=2048, p=0.1, residual=True),
        # The gradient of a small policy that is trained in single precision.
        dict(name="drop_odd", form="drop", type="f32", B=16, L=255, D=129, p=0.25, residual=False),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    form = rng.choice(["step", "delta", "delta", "train", "train", "norm", "grad", "drop"])
    c = {"form": form, "type": rng.choice(["bf16", "bf16", "f32"])}
    if form in ("step", "delta", "train"):
        H = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
        shared = [n for n in range(1, H + 1) if H % n == 0 and n * 4 >= H]
        few = rng.choice(shared)                                                     # heads that are shared, of ...
        Q, K, V = rng.choice([(H, H, H), (few, few, H), (H, few, few), (H, H, few)])
        size = lambda: rng.choice([32, 64, 64, 128, 128, _spread(rng, 16, 128)])     # noqa: E731
        c.update(H=H, Q=Q, K=K, V=V, dk=size(), dv=size())
        if form == "step":
            c["B"] = _spread(rng, 1, max(1, (512 * 16 * 128 * 128) // (H * c["dk"] * c["dv"]) // 4))
        else:
            # values in the batch: up to half the largest listed case's, a quarter for gradients and in single precision
            most = (1 << 26) // (H * max(c["dk"], c["dv"])) // (4 if form == "train" else 1) // (2 if c["type"] == "f32" else 1)
            c["L"] = _spread(rng, 1, min(most, 16384))
            c["B"] = _spread(rng, 1, max(1, min(256, most // c["L"])))
            c["ragged"] = rng.random() < 0.5
        return c
    c["D"] = rng.choice([256, 512, 1024, 2048, 4096, _spread(rng, 16, 8192), _spread(rng, 16, 8192)])
    most = (1 << 25) // c["D"]
    c["L"] = _spread(rng, 1, min(most, 16384))
    c["B"] = _spread(rng, 1, max(1, min(512, most // c["L"])))
    if form == "drop":
        c.update(p=rng.choice([0.05, 0.1, 0.2, 0.5]), residual=rng.random() < 0.5)
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
class _State:
    pass


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1))
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    s = _State()
    s.form, s.type = case["form"], DTYPES[case["type"]]
    B, L = case["B"], case.get("L", 1)
    if s.form in ("step", "delta", "train"):
        H, dk, dv = case["H"], case["dk"], case["dv"]
        unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
        s.q, s.k = (unit(normal(B, L, n, dk)).to(s.type) for n in (case["Q"], case["K"]))
        s.v = normal(B, L, case["V"], dv).to(s.type)
        # decays and strengths as a projection of each token gives them: a rate for each head, from slow to fast, times a positive gate
        rate = 0.02 * torch.exp2(torch.arange(H, device="cuda", dtype=torch.float32) * (5.0 / H))
        s.log_decay = -rate * torch.nn.functional.softplus(normal(B, L, H))
        s.beta = torch.sigmoid(normal(B, L, H))
        s.scale = dk ** -0.5
        s.state = 0.3 * normal(B, H, dk, dv)
        s.lengths = None
        if case.get("ragged"):
            s.lengths = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s.lengths[0] = L
        if s.form == "train":
            s.dout, s.dstate = normal(B, L, H, dv).to(s.type), 0.3 * normal(B, H, dk, dv)
        return s
    D = case["D"]
    s.x = (normal(B, L, D) * (1.0 + normal(B, L, 1).abs()) + 0.5 * normal(D)).to(s.type)   # rows of unlike sizes, off their middle
    if s.form == "drop":
        s.p, s.seed, s.offset = case["p"], 0x9E3779B97F4A7C15 ^ (seed * 0x1_0000_0001), 7 * seed + (1 << 33)
        s.residual = normal(B, L, D).to(s.type) if case["residual"] else None
        return s
    s.weight, s.bias = 1.0 + 0.1 * normal(D), 0.1 * normal(D)
    if s.form == "grad":
        s.dout = normal(B, L, D).to(s.type)
    return s


# -------------------------------------------------------------------------------------------------------- plain forms
CHUNK = 64


def _heads(t, H):
    """[B, L, n, d] in any type -> [B, H, L, d] in 32 bits, shared heads repeated."""
    t = t.float().transpose(1, 2)
    return t if t.shape[1] == H else t.repeat_interleave(H // t.shape[1], 1)


def _inverse(a):
    """(1 + a)^-1 of strictly lower triangular matrices, by halves: two products for each doubling of the blocks."""
    n = a.shape[-1]
    at = torch.arange(n, device=a.device)
    t, half = torch.eye(n, device=a.device), 1
    while half < n:
        below = (at[:, None] // (2 * half) == at // (2 * half)) & (at[:, None] // half > at // half)
        t = t - torch.matmul(torch.matmul(t, a * below), t)
        half *= 2
    return t


def _plain_delta(q, k, v, log_decay, beta, state, lengths, scale):
    """Within pieces of the sequence by the products of all pairs (what the tokens of a piece write depends on what those before them
    wrote: a triangular system), between them by the state.  Rows [B, L, n, d] in 32 bits, results [B, L, H, dv] and [B, H, dk, dv]."""
    B, L, H = beta.shape
    q, k, v = (_heads(t, H) for t in (q, k, v))
    g, b = log_decay.double().transpose(1, 2), beta.transpose(1, 2)
    if lengths is not None:
        here = (torch.arange(L, device=q.device) < lengths[:, None])[:, None]
        q, k, v = (t.masked_fill(~here[..., None], 0) for t in (q, k, v))
        g, b = g.masked_fill(~here, 0), b.masked_fill(~here, 0)
    size = min(CHUNK, 1 << (L - 1).bit_length())
    n = -(-L // size)
    q, k, v = (torch.nn.functional.pad(t, (0, 0, 0, n * size - L)).reshape(B, H, n, size, -1) for t in (q, k, v))
    g, b = (torch.nn.functional.pad(t, (0, n * size - L)).reshape(B, H, n, size) for t in (g, b))
    at = torch.arange(size, device=q.device)
    sums = g.cumsum(-1)
    gap = (sums[..., :, None] - sums[..., None, :]).masked_fill(at[:, None] < at, -math.inf).exp().float()
    pairs = b[..., None] * gap * torch.matmul(k, k.transpose(-1, -2))
    solve = _inverse(pairs.masked_fill(at[:, None] <= at, 0))
    since, left = sums.exp().float()[..., None], (sums[..., -1:] - sums).exp().float()[..., None]
    reads, writes = torch.matmul(solve, b[..., None] * since * k), torch.matmul(solve, b[..., None] * v)
    seen, asks, into = scale * gap * torch.matmul(q, k.transpose(-1, -2)), scale * since * q, (left * k).transpose(-1, -2)
    out = []
    for i in range(n):
        u = writes[:, :, i] - torch.matmul(reads[:, :, i], state)
        out.append(torch.matmul(asks[:, :, i], state) + torch.matmul(seen[:, :, i], u))
        state = since[:, :, i, -1:] * state + torch.matmul(into[:, :, i], u)
    return torch.cat(out, 2)[:, :, :L].transpose(1, 2), state


def _plain_train(s):
    leaves = [t.detach().float().requires_grad_() for t in (s.q, s.k, s.v, s.log_decay, s.beta, s.state)]
    with torch.enable_grad():
        results = _plain_delta(*leaves, s.lengths, s.scale)
    grads = torch.autograd.grad(results, leaves, (s.dout.float(), s.dstate))
    return [t.to(s.type) for t in grads[:3]] + list(grads[3:])


def _plain_step(s):
    H = s.beta.shape[2]
    q, k, v = (_heads(t, H)[:, :, 0] for t in (s.q, s.k, s.v))
    state = s.state * torch.exp(s.log_decay[:, 0])[..., None, None]
    u = s.beta[:, 0, :, None] * (v - torch.matmul(k[..., None, :], state)[..., 0, :])
    s.state = state + k[..., None] * u[..., None, :]
    out = torch.matmul(q[..., None, :], s.state)[..., 0, :] * s.scale
    return [out[:, None].to(s.type), s.state]


def _normed(x):
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _random(blocks, seed, offset, device):
    """Philox4x32-10: of counters (block, offset) and the key ``seed`` four words of 32 bits each, [blocks, 4] in 64 bits."""
    low, block = 0xFFFFFFFF, torch.arange(blocks, device=device, dtype=torch.int64)
    c = [block & low, block >> 32, torch.full_like(block, offset & low), torch.full_like(block, offset >> 32)]
    key = [seed & low, seed >> 32 & low]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57          # (64 bits that run over keep the upper words, as a shift and a mask take them)
        c = [(b >> 32 & low) ^ c[1] ^ key[0], b & low, (a >> 32 & low) ^ c[3] ^ key[1], a & low]
        key = [key[0] + 0x9E3779B9 & low, key[1] + 0xBB67AE85 & low]
    return torch.stack(c, 1)


def _kept(shape, p, seed, offset, device):
    """Which elements stay, and what they are multiplied with: element i has the 16 bits i % 8 of block i / 8."""
    n, border = math.prod(shape), int(p * 65536 + 0.5)
    words = _random(-(-n // 8), seed, offset, device)
    halves = torch.stack((words & 0xFFFF, words >> 16), -1).flatten()[:n]
    return (halves >= border).reshape(shape), 65536.0 / (65536 - border)


def _plain(s):
    if s.form == "step":
        return _plain_step(s)
    if s.form == "delta":
        out, state = _plain_delta(s.q, s.k, s.v, s.log_decay, s.beta, s.state, s.lengths, s.scale)
        return [out.to(s.type), state]
    if s.form == "train":
        return _plain_train(s)
    x = s.x.float()
    if s.form == "norm":
        return [(_normed(x)[0] * s.weight + s.bias).to(s.type)]
    if s.form == "drop":
        keep, factor = _kept(x.shape, s.p, s.seed, s.offset, x.device)
        out = torch.where(keep, x * factor, 0.0)
        return [(out if s.residual is None else s.residual.float() + out).to(s.type)]
    xh, r = _normed(x)
    dout = s.dout.float()
    h = dout * s.weight
    dx = r * (h - h.mean(-1, keepdim=True) - xh * (h * xh).mean(-1, keepdim=True))
    return [dx.to(s.type), (dout * xh).sum((0, 1)), dout.sum((0, 1))]


# --------------------------------------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return _plain(s)
    from paper_2311_09445_amd import sequence as seq
    if s.form == "step":
        return [seq.gated_delta_step(s.q, s.k, s.v, s.log_decay, s.beta, s.state, scale=s.scale), s.state]
    if s.form == "delta":
        return list(seq.gated_delta(s.q, s.k, s.v, s.log_decay, s.beta, s.state, lengths=s.lengths, scale=s.scale))
    if s.form == "train":
        return list(seq.gated_delta_backward(s.dout, s.q, s.k, s.v, s.log_decay, s.beta, s.state, dstate=s.dstate,
                                             lengths=s.lengths, scale=s.scale))
    if s.form == "norm":
        return [seq.layer_norm(s.x, s.weight, s.bias, eps=EPS)]
    if s.form == "grad":
        return list(seq.layer_norm_backward(s.dout, s.x, s.weight, eps=EPS))
    return [seq.dropout(s.x, s.p, s.seed, s.offset, residual=s.residual)]


# ------------------------------------------------------------------------------------------- what a pass cannot spare
def work(case):
    """Bytes: every input read once, every output written once.  Operations: of the recurrent form, two products with the state and a sum
    into it for each token and head (the gradient: two states, seven such); of the norm some eight for each value, twice that for its gradient."""
    B, L, e = case["B"], case.get("L", 1), 2 if case["type"] == "bf16" else 4
    if case["form"] in ("step", "delta", "train"):
        H, dk, dv = case["H"], case["dk"], case["dv"]
        rows, out = B * L * ((case["Q"] + case["K"]) * dk + case["V"] * dv) * e, B * L * H * dv * e
        gates, states = 8 * B * L * H, 4 * B * H * dk * dv
        if case["form"] == "train":
            return {"bytes": 2 * rows + out + 2 * gates + 3 * states, "flops": 14 * B * L * H * dk * dv}
        return {"bytes": rows + out + gates + 2 * states, "flops": 6 * B * L * H * dk * dv}
    n = B * L * case["D"]
    tensors = 2 + (case["form"] == "grad") + bool(case.get("residual"))
    return {"bytes": n * e * tensors, "flops": n * {"norm": 8, "grad": 16, "drop": 2}[case["form"]]}


# ------------------------------------------------------------------------------- the definition, token by token in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if s.form in ("step", "delta", "train"):
        return _exact_delta(s)
    x = s.x.to(f64)
    if s.form == "drop":
        keep, _ = _kept(x.shape, s.p, s.seed, s.offset, x.device)
        out = x * keep / (1.0 - int(s.p * 65536 + 0.5) / 65536)
        return [out if s.residual is None else out + s.residual.to(f64)]
    middle = x.sum(-1, keepdim=True) / x.shape[-1]
    spread = ((x - middle).pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
    if s.form == "norm":
        return [(x - middle) / spread * s.weight.to(f64) + s.bias.to(f64)]
    y, dout = (x - middle) / spread, s.dout.to(f64)
    h = dout * s.weight.to(f64)
    dx = (h - h.sum(-1, keepdim=True) / x.shape[-1] - y * (h * y).sum(-1, keepdim=True) / x.shape[-1]) / spread
    return [dx, (dout * y).sum((0, 1)), dout.sum((0, 1))]


def _exact_delta(s):
    """The recurrence and, against time, that of the state's gradient, a token at a time."""
    f64 = torch.float64
    B, L, H = s.beta.shape
    many = lambda t: t.to(f64).repeat_interleave(H // t.shape[2], 2).unbind(1)  # noqa: E731
    q, k, v = many(s.q), many(s.k), many(s.v)
    a, beta = s.log_decay.to(f64).exp()[..., None].unbind(1), s.beta.to(f64)[..., None].unbind(1)
    length = torch.full((B,), L, device=s.q.device) if s.lengths is None else s.lengths
    ragged = s.lengths is not None
    valid = torch.arange(L, device=s.q.device) < length[:, None]                     # [B, L]
    here, mask = valid[..., None, None, None].unbind(1), valid[..., None]
    read = lambda S, x: torch.matmul(x[..., None, :], S)[..., 0, :]                  # noqa: E731    x^T S
    back = lambda S, x: torch.matmul(S, x[..., None])[..., 0]                        # noqa: E731    S x

    def forward(visit):
        """Calls visit(t, state the token sees decayed, what it writes, state behind it)."""
        S = s.state.to(f64)
        for t in range(L):
            D = S * a[t][..., None]
            u = beta[t] * (v[t] - read(D, k[t]))
            new = torch.addcmul(D, k[t][..., None], u[..., None, :])
            visit(t, D, u, new)
            S = torch.where(here[t], new, S) if ragged else new
        return S

    if s.form != "train":
        out = []
        last = forward(lambda t, D, u, S: out.append(s.scale * read(S, q[t])))
        return [torch.stack(out, 1) * mask[..., None], last]
    do = s.dout.to(f64).unbind(1)
    us, dqs, outs = [], [], []
    last = forward(lambda t, D, u, S: (us.append(u), dqs.append(s.scale * back(S, do[t])), outs.append(s.scale * read(S, q[t]))))
    R = s.dstate.to(f64)
    dus, dwrite = [None] * L, [None] * L
    for t in range(L - 1, -1, -1):
        E = torch.addcmul(R, q[t][..., None], do[t][..., None, :], value=s.scale)     # of the state behind token t
        dus[t] = read(E, k[t])
        dwrite[t] = back(E, us[t])
        E = torch.addcmul(E, k[t][..., None], (beta[t] * dus[t])[..., None, :], value=-1.0) * a[t][..., None]
        R = torch.where(here[t], E, R) if ragged else E
    dread, values = [], []
    forward(lambda t, D, u, S: (dread.append(-back(D, beta[t] * dus[t])), values.append(v[t] - read(D, k[t]))))
    stack = lambda ts: torch.stack(ts, 1) * mask[..., None]                          # noqa: E731
    fold = lambda t, n: t.reshape(B, L, n, H // n, -1).sum(3)                        # noqa: E731
    dv = stack(dus) * s.beta.to(f64)[..., None]
    # the size of a state that a token sees does not matter but for what is read of it and written to it, here and later
    change = (stack(outs) * s.dout.to(f64)).sum(-1) - (dv * s.v.to(f64).repeat_interleave(H // s.v.shape[2], 2)).sum(-1)
    dg = (change.flip(1).cumsum(1).flip(1) + (last * s.dstate.to(f64)).sum((-1, -2))[:, None]) * mask
    return [fold(stack(dqs), s.q.shape[2]), fold(stack(dwrite) + stack(dread), s.k.shape[2]), fold(dv, s.v.shape[2]), dg,
            (stack(dus) * stack(values)).sum(-1), R]
