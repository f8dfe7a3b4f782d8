"""Timed work of the sequence operators: what a learner of replayed sequences, and the actors beside it, have them do.

A *case* is a dict of plain values.  ``prepare`` makes what such a program has in hand, ``run`` is one pass through one
operator, ``work`` the bytes and operations that pass cannot do without, ``exact`` its outputs from the definition in
64 bits.  ``own`` says whether ``run`` takes the framework's operators or the plain form written here.

Forms (``"form"``):
  step    linear attention with a decay for each head, one token of many actors: the states are updated in place
  attend  the same over sequences (ragged where ``ragged``), from given states: outputs and final states
  train   its gradient: of queries, keys, values and initial states
  rotate  rotary positions alone: half or interleaved pairs, part of the head, scaled frequencies
  norm    norms of queries and keys for each head, with the rotation in the same pass
  grad    the gradient of that: of queries, keys and both weights
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # 64 actors stepping together, a small recurrent policy: nothing but latency.
        dict(name="step_actors", form="step", type="bf16", B=64, H=4, G=4, dk=64, dv=64),
        # A fleet of 1024 environments with a large policy: a gigabyte of states read and written for one token each.
        dict(name="step_fleet", form="step", type="bf16", B=1024, H=16, G=16, dk=128, dv=128),
        # A learner's batch of replayed stretches of up to 80 steps, each from its stored state, some cut short by an episode's end.
        dict(name="attend_replay", form="attend", type="bf16", B=64, L=80, H=4, G=4, dk=64, dv=64, ragged=True),
        # Nothing here is a power of two: single precision, heads that share keys and values.
        dict(name="attend_odd", form="attend", type="f32", B=3, L=1001, H=6, G=2, dk=48, dv=80, ragged=True),
        # One whole history of 65536 steps through a large policy: few rows, a long axis.
        dict(name="attend_long", form="attend", type="bf16", B=1, L=65536, H=16, G=16, dk=128, dv=128, ragged=False),
        # The gradient for a batch of 32 replayed stretches of up to 512 steps; eight heads share two of keys and values.
        dict(name="train_replay", form="train", type="bf16", B=32, L=512, H=8, G=2, dk=64, dv=64, ragged=True),
        # The gradient through two long histories.
        dict(name="train_long", form="train", type="bf16", B=2, L=16384, H=16, G=16, dk=128, dv=128, ragged=False),
        # The gradient of a small policy that is trained in single precision.
        dict(name="train_single", form="train", type="f32", B=16, L=256, H=4, G=4, dk=32, dv=32, ragged=False),
        # Rotary positions of 32 actors' queries at far positions.
        dict(name="rotate_actors", form="rotate", type="f32", B=32, L=1, H=8, D=64, rot=64, layout="half", far=1 << 20, scale=1.0),
        # Rotary positions over long stretches: half of each head, interleaved, frequencies slowed down by eight.
        dict(name="rotate_long", form="rotate", type="bf16", B=4, L=8192, H=32, D=128, rot=64, layout="interleaved", far=1 << 17, scale=8.0),
        # Queries and keys of a learner's batch.
        dict(name="norm_learner", form="norm", type="bf16", B=16, L=2048, H=32, G=8, D=128, rot=128, layout="half", far=4096, scale=1.0),
        # Their gradient, on heads and stretches of odd sizes.
        dict(name="grad_odd", form="grad", type="bf16", B=8, L=1023, H=16, G=4, D=96, rot=48, layout="half", far=4096, scale=1.0),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    form = rng.choice(["step", "attend", "attend", "train", "train", "rotate", "norm", "grad"])
    c = {"form": form, "type": rng.choice(["bf16", "bf16", "f32"])}
    G = rng.choice([1, 2, 4, 8, 16])
    H = G * rng.choice([1, 1, 1, 2, 4]) if G < 8 else G
    if form in ("step", "attend", "train"):
        size = lambda: rng.choice([32, 64, 64, 128, 128, _spread(rng, 16, 128)])  # noqa: E731
        c.update(H=H, G=G, dk=size(), dv=size())
        if form == "step":
            c["B"] = _spread(rng, 1, max(1, (1024 * 16 * 128 * 128) // (H * c["dk"] * c["dv"]) // 4))
        else:
            # values in the batch: up to half the largest listed case's, a quarter for gradients and in single precision
            most = (1 << 26) // (H * max(c["dk"], c["dv"])) // (2 if form == "train" else 1) // (2 if c["type"] == "f32" else 1)
            c["L"] = _spread(rng, 1, min(most, 32768))
            c["B"] = _spread(rng, 1, max(1, min(256, most // c["L"])))
            c["ragged"] = rng.random() < 0.5
    else:
        D = rng.choice([32, 64, 64, 128, 128, 80, 96])
        c.update(H=H, D=D, rot=rng.choice([D, D, D // 2]), layout=rng.choice(["half", "interleaved"]),
                 far=rng.choice([1, 4096, 1 << 17, 1 << 20]), scale=rng.choice([1.0, 1.0, 4.0, 8.0]))
        if form != "rotate":
            c["G"] = G
        most = (1 << 26) // (2 * H * D)
        c["L"] = _spread(rng, 1, min(most, 16384))
        c["B"] = _spread(rng, 1, max(1, min(512, most // c["L"])))
    return c


# ------------------------------------------------------------------------------------------------------------ inputs
class _State:
    pass


def _frequencies(case):
    """rot/2 frequencies of base 10000, all slowed down by ``scale`` (positions of a longer stretch fall between those
    trained on), and the magnitude that the rotated pairs are multiplied with."""
    n = case["rot"] // 2
    f = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) / case["scale"]
    return f.float(), 1.0 if case["scale"] == 1.0 else 0.1 * math.log(case["scale"]) + 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * (seed + 1))
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    s = _State()
    s.form, s.type = case["form"], DTYPES[case["type"]]
    B, H, L = case["B"], case["H"], case.get("L", 1)
    if s.form in ("step", "attend", "train"):
        G, dk, dv = case["G"], case["dk"], case["dv"]
        # queries and keys as a norm leaves them; decays from fast to slow over the heads, as policies of this kind fix them
        s.q, s.k, s.v = normal(B, L, H, dk).to(s.type), normal(B, L, G, dk).to(s.type), normal(B, L, G, dv).to(s.type)
        s.log_decay = -torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda", dtype=torch.float32) / H)
        s.scale = dk ** -0.5
        s.state = normal(B, H, dk, dv)
        s.lengths = None
        if case.get("ragged"):
            s.lengths = torch.randint(0, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s.lengths[0] = L
        if s.form == "train":
            s.dout, s.dstate = normal(B, L, H, dv).to(s.type), normal(B, H, dk, dv)
        return s
    D = case["D"]
    s.freqs, s.magnitude = _frequencies(case)
    s.freqs = s.freqs.cuda()
    s.layout = case["layout"]
    start = torch.randint(0, case["far"], (B, 1), generator=g, device="cuda", dtype=torch.int32)
    s.positions = start + torch.arange(L, device="cuda", dtype=torch.int32)
    s.q = normal(B, L, H, D).to(s.type)
    if s.form != "rotate":
        s.k = normal(B, L, case["G"], D).to(s.type)
        s.qw, s.kw = 1.0 + 0.1 * normal(D), 1.0 + 0.1 * normal(D)
    if s.form == "grad":
        s.dq, s.dk = normal(B, L, H, D).to(s.type), normal(B, L, case["G"], D).to(s.type)
    return s


# -------------------------------------------------------------------------------------------------------- plain forms
CHUNK = 128


def _decayed(x, y, z, log_decay, state, scale, back):
    """Rows of a decayed product of all pairs, on [B, H, L, .]: out[i] = sum over j <= i of decay^(i-j) scale (x[i].y[j]) z[j], and
    what the state at the start adds.  Within pieces of the sequence by the products of all pairs, between them by the states at their
    starts.  Against time (``back``) the state is that of a gradient: the scale is in what it sums, and it has been decayed once more."""
    B, H, L, dx = x.shape
    dz = z.shape[-1]
    size = min(CHUNK, L)
    n = -(-L // size)
    x, y, z = (torch.nn.functional.pad(t, (0, 0, 0, n * size - L)).reshape(B, H, n, size, -1) for t in (x, y, z))
    at = torch.arange(size, device=x.device, dtype=torch.float32)
    g = log_decay[:, None]
    gap = at[:, None] - at
    inside = torch.exp(gap.clamp(min=0) * g[..., None]) * (gap >= 0)                          # [H, C, C]
    out = torch.matmul(torch.matmul(x, y.transpose(-1, -2)) * (scale * inside[:, None]), z)
    into = torch.exp((size - 1 - at + back) * g) * (scale if back else 1.0)
    grown = torch.matmul((y * into[:, None, :, None]).transpose(-1, -2), z)
    piece = torch.arange(n, device=x.device, dtype=torch.float32)
    gap = piece[:, None] - 1 - piece
    between = torch.exp(gap.clamp(min=0) * size * g[..., None]) * (gap >= 0)                 # [H, n, n]
    starts = torch.matmul(between, grown.reshape(B, H, n, dx * dz)).reshape(B, H, n, dx, dz)
    starts = starts + torch.exp(piece * size * g)[..., None, None] * state[:, :, None]
    outof = torch.exp((at + 1 - back) * g) * (1.0 if back else scale)
    out = out + torch.matmul(x, starts) * outof[:, None, :, None]
    return out.reshape(B, H, n * size, dz)[:, :, :L]


def _total(y, z, log_decay, state, lengths, scale, back):
    """The state behind the last token (against time: the gradient of the state before the first)."""
    left = lengths[:, None, None] - 1 - torch.arange(y.shape[2], device=y.device)             # [B, 1, L]
    w = torch.exp((left.clamp(min=0) + back) * log_decay[:, None]) * (left >= 0) * (scale if back else 1.0)
    kept = torch.exp(lengths[:, None] * log_decay)
    return torch.matmul((y * w[..., None]).transpose(-1, -2), z) + kept[..., None, None] * state


def _heads(t, H):
    """[B, L, G, d] in any type -> [B, H, L, d] in 32 bits, shared heads repeated."""
    t = t.float().transpose(1, 2)
    return t if t.shape[1] == H else t.repeat_interleave(H // t.shape[1], 1)


def _lengths(s):
    B, L = s.q.shape[:2]
    return torch.full((B,), L, device=s.q.device) if s.lengths is None else s.lengths


def _valid(s):
    return (torch.arange(s.q.shape[1], device=s.q.device) < _lengths(s)[:, None])[:, None, :, None]


def _fold(t, G):
    """[B, H, L, d] -> [B, L, G, d]: the gradients of the heads that share one are added up."""
    B, H, L, d = t.shape
    return t.reshape(B, G, H // G, L, d).sum(2).transpose(1, 2)


def _plain_attend(s):
    H = s.q.shape[2]
    here = _valid(s)
    q, k, v = (_heads(t, H).masked_fill(~here, 0) for t in (s.q, s.k, s.v))
    out = _decayed(q, k, v, s.log_decay, s.state, s.scale, 0).masked_fill(~here, 0)
    return [out.transpose(1, 2).to(s.type), _total(k, v, s.log_decay, s.state, _lengths(s), s.scale, 0)]


def _plain_train(s):
    H, G, L = s.q.shape[2], s.k.shape[2], s.q.shape[1]
    here, lengths = _valid(s), _lengths(s)
    q, k, v, do = (_heads(t, H).masked_fill(~here, 0) for t in (s.q, s.k, s.v, s.dout))
    dq = _decayed(do, v, k, s.log_decay, s.state.transpose(-1, -2), s.scale, 0).masked_fill(~here, 0)
    # the gradients of keys and values run against time: the valid part of each sequence is turned around, and back
    turn = (lengths[:, None] - 1 - torch.arange(L, device=q.device)).clamp(min=0)[:, None, :, None].long()
    q, k, v, do = (torch.take_along_dim(t, turn, 2).masked_fill(~here, 0) for t in (q, k, v, do))
    dv = _decayed(k, q, do, s.log_decay, s.dstate, s.scale, 1)
    dk = _decayed(v, do, q, s.log_decay, s.dstate.transpose(-1, -2), s.scale, 1)
    dk, dv = (_fold(torch.take_along_dim(t, turn, 2).masked_fill(~here, 0), G).to(s.type) for t in (dk, dv))
    return [dq.transpose(1, 2).to(s.type), dk, dv, _total(q, do, s.log_decay, s.dstate, lengths, s.scale, 1)]


def _rotated(x, s, back=False):
    """Rotary positions on [B, L, H, D] in 32 bits.  The angles are reduced in 64 bits: at position 2^20 an angle in 32 bits is
    off by 0.06."""
    half = s.freqs.numel()
    angle = s.positions.double()[..., None, None] * s.freqs.double()
    c, n = ((s.magnitude * t).float() for t in (torch.cos(angle), torch.sin(angle)))
    n = -n if back else n
    if s.layout == "half":
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * c - b * n, a * n + b * c), -1)
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * c - b * n, a * n + b * c), -1).flatten(-2)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _normed(x):
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _norm_gradient(x, w, dout, s):
    xh, r = _normed(x.float())
    dy = _rotated(dout.float(), s, back=True)
    h = dy * w
    dx = r * (h - xh * (h * xh).mean(-1, keepdim=True))
    return dx.to(s.type), (dy * xh).sum((0, 1, 2))


def _plain(s):
    if s.form == "step":
        H = s.q.shape[2]
        q, k, v = (_heads(t, H)[:, :, 0] for t in (s.q, s.k, s.v))
        s.state = s.state * torch.exp(s.log_decay)[:, None, None] + k[..., None] * v[..., None, :]
        out = torch.matmul(q[..., None, :], s.state)[..., 0, :] * s.scale
        return [out[:, None].to(s.type), s.state]
    if s.form == "attend":
        return _plain_attend(s)
    if s.form == "train":
        return _plain_train(s)
    if s.form == "rotate":
        return [_rotated(s.q.float(), s).to(s.type)]
    if s.form == "norm":
        return [_rotated(_normed(x.float())[0] * w, s).to(s.type) for x, w in ((s.q, s.qw), (s.k, s.kw))]
    (dq, dqw), (dk, dkw) = (_norm_gradient(x, w, d, s) for x, w, d in ((s.q, s.qw, s.dq), (s.k, s.kw, s.dk)))
    return [dq, dk, dqw, dkw]


# --------------------------------------------------------------------------------------------------------- one pass
def run(s):
    if not own:
        return _plain(s)
    from paper_2311_09445_amd import sequence as seq
    if s.form == "step":
        return [seq.linear_attention_step(s.q, s.k, s.v, s.log_decay, s.state, scale=s.scale), s.state]
    if s.form == "attend":
        return list(seq.linear_attention(s.q, s.k, s.v, s.log_decay, s.state, lengths=s.lengths, scale=s.scale))
    if s.form == "train":
        return list(seq.linear_attention_backward(s.dout, s.q, s.k, s.v, s.log_decay, s.state, dstate=s.dstate,
                                                  lengths=s.lengths, scale=s.scale))
    turn = dict(layout=s.layout, magnitude=s.magnitude)
    if s.form == "rotate":
        return [seq.rotate(s.q, s.positions, s.freqs, **turn)]
    if s.form == "norm":
        return list(seq.norm_rotate(s.q, s.k, s.qw, s.kw, s.positions, s.freqs, eps=EPS, **turn))
    return list(seq.norm_rotate_backward(s.dq, s.dk, s.q, s.k, s.qw, s.kw, s.positions, s.freqs, eps=EPS, **turn))


# ------------------------------------------------------------------------------------------- what a pass cannot spare
def work(case):
    """Bytes: every input read once, every output written once.  Operations: of the recurrent form, a product with the state and a sum
    into it for each token and head (the gradient: two states, three products); of the rotation and the norm some ten for each value."""
    B, H, L, e = case["B"], case["H"], case.get("L", 1), 2 if case["type"] == "bf16" else 4
    if case["form"] in ("step", "attend", "train"):
        G, dk, dv = case["G"], case["dk"], case["dv"]
        rows, states = B * L * (H + G) * (dk + dv) * e, 4 * B * H * dk * dv
        if case["form"] == "train":
            return {"bytes": 2 * rows - B * L * H * dv * e + 3 * states, "flops": 10 * B * L * H * dk * dv}
        return {"bytes": rows + 2 * states, "flops": 4 * B * L * H * dk * dv}
    heads = H if case["form"] == "rotate" else H + case["G"]
    n = B * L * heads * case["D"]
    return {"bytes": n * e * (3 if case["form"] == "grad" else 2) + 4 * B * L, "flops": n * {"rotate": 3, "norm": 7, "grad": 14}[case["form"]]}


# ------------------------------------------------------------------------------- the definition, token by token in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if s.form in ("step", "attend", "train"):
        return _exact_recurrence(s)
    out = [_exact_head(s, s.q, getattr(s, "qw", None), getattr(s, "dq", None))]
    if s.form != "rotate":
        out.append(_exact_head(s, s.k, s.kw, getattr(s, "dk", None)))
    return [t for pair in zip(*out) for t in pair] if s.form == "grad" else [t[0] for t in out]


def _exact_recurrence(s):
    f64 = torch.float64
    B, L, H, dk = s.q.shape
    G, dv = s.v.shape[2:]
    head = torch.arange(H, device=s.q.device) // (H // G)
    decay = torch.exp(s.log_decay.to(f64))[None, :, None, None]
    lengths = [L] * B if s.lengths is None else s.lengths.tolist()
    q, do = s.q.to(f64).unbind(1), None if s.form != "train" else s.dout.to(f64).unbind(1)
    k, v = s.k.to(f64).unbind(1), s.v.to(f64).unbind(1)
    ragged = min(lengths) < L
    length = torch.tensor(lengths, device=s.q.device)[:, None, None, None]

    def col(t):
        return t[:, head, :, None] if t.shape[1] != H else t[..., None]

    def row(t):
        return t[:, head, None, :] if t.shape[1] != H else t[:, :, None, :]

    out, dq, state = [], [], s.state.to(f64)
    for t in range(L):
        new = torch.addcmul(state * decay, col(k[t]), row(v[t]))
        state = torch.where(length > t, new, state) if ragged else new
        if s.form == "train":
            dq.append(torch.matmul(state, do[t][..., None])[..., 0])
        else:
            out.append(torch.matmul(q[t][:, :, None], state)[:, :, 0])
    here = torch.arange(L, device=s.q.device)[:, None, None] < length
    if s.form != "train":
        return [s.scale * torch.stack(out, 1).masked_fill(~here, 0), state]
    back, dks, dvs = s.dstate.to(f64), [], []       # ``back``: of the state behind token t, without what token t itself brings
    for t in range(L - 1, -1, -1):
        at = torch.addcmul(back, col(q[t]), row(do[t]), value=s.scale)
        dks.append(torch.matmul(at, row(v[t]).transpose(-1, -2))[..., 0])
        dvs.append(torch.matmul(col(k[t]).transpose(-1, -2), at)[..., 0, :])
        back = torch.where(length > t, at * decay, back) if ragged else at * decay
    share = lambda ts: torch.stack(ts[::-1], 1).masked_fill(~here, 0).reshape(B, L, G, H // G, -1).sum(3)  # noqa: E731
    return [s.scale * torch.stack(dq, 1).masked_fill(~here, 0), share(dks), share(dvs), back]


def _exact_head(s, x, w, dout):
    """(rows,) or, with ``dout``, (gradient of rows, gradient of weight): the rotation as a product of complex numbers."""
    x = x.double()
    rot, D = 2 * s.freqs.numel(), x.shape[-1]
    unit = torch.polar(torch.full((), s.magnitude, dtype=torch.float64, device=x.device), s.positions.double()[..., None] * s.freqs.double())[:, :, None]

    def turned(t, by):
        pairs = t[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2) if s.layout == "half" else t[..., :rot].unflatten(-1, (rot // 2, 2))
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
        pairs = pairs.transpose(-1, -2) if s.layout == "half" else pairs
        return torch.cat((pairs.flatten(-2), t[..., rot:]), -1)

    if w is None:
        return (turned(x, unit),)
    w = w.double()
    spread = (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt()
    if dout is None:
        return (turned(x / spread * w, unit),)
    dy = turned(dout.double(), unit.conj())
    along = (dy * w * x).sum(-1, keepdim=True) / (D * spread.pow(3))
    return dy * w / spread - x * along, (dy * x / spread).sum((0, 1, 2))
