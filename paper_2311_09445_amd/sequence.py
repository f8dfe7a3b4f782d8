"""Sequence operators of ``libper_hip.so`` (the C-ABI declared in ``include/per_seq.h``): what a learner of replayed
sequences, and the actors beside it, run on the rows that ``per.PrioritizedReplay`` samples.

Rows are device tensors [batch, length, heads, width] in bfloat16 or float32; every stride is taken as it is, but the last
dimension has to be contiguous.  Work is enqueued on the current stream; nothing synchronises.  Tensors are taken apart, and
results allocated, in ``_seq_binding.so`` (``csrc/seq_binding.cpp``: the checks and their messages are there).

Inputs that ask for a gradient get one: the calls of sequences are then nodes of torch's graph (with no tensors given for their
results, which could not be).  Gradients of gradients are refused but for the rotation's, and so are gradients of decays and frequencies;
the calls that form gradients, and single tokens, are no nodes.

There is no CPU fallback.
"""
from __future__ import annotations

import math
import os

from . import per
from .per import PerError

_HERE = os.path.dirname(os.path.abspath(__file__))
BINDING_PATH = os.path.join(_HERE, "_seq_binding.so")

EXPORTS = [
    "per_rotate", "per_norm_rotate", "per_norm_rotate_workspace", "per_norm_rotate_backward", "per_linear_attention_workspace",
    "per_linear_attention", "per_linear_attention_backward", "per_linear_attention_step",
]
LAYOUTS = {"half": 0, "interleaved": 1}

_CALLS = None


def _calls():
    global _CALLS
    if _CALLS is None:
        import torch  # noqa: F401  (its libraries must be loaded before the binding)
        per._lib()
        if not os.path.exists(BINDING_PATH):
            raise ImportError(f"{BINDING_PATH} is missing: build it with `python -m paper_2311_09445_amd.build`.")
        from . import _seq_binding
        _CALLS = _seq_binding
    return _CALLS


def _layout(layout):
    try:
        return LAYOUTS[layout]
    except (KeyError, TypeError):
        raise ValueError(f"layout must be one of {sorted(LAYOUTS)}, got {layout!r}") from None


# ------------------------------------------------------------------------------------------------------ rotary positions
def rotary_frequencies(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: int = 0,
                       fast: float = 32.0, slow: float = 1.0, device="cuda"):
    """(freqs, magnitude) for ``rotate`` and ``norm_rotate``: rot/2 frequencies base^(-2p/rot) in fp32, for stretches
    ``factor`` times as long as those trained on:

    ``none``    as they are
    ``linear``  all slowed down by ``factor``
    ``base``    a larger base, base * factor^(rot/(rot-2)): the slowest pair is slowed down by ``factor``, the fastest not at all
    ``parts``   pairs that turn more than ``fast`` times within ``trained`` tokens stay, those that turn less than ``slow``
                times are slowed down by ``factor``, in between the two are mixed; the magnitude grows with 0.1 ln(factor)
    """
    import torch
    if rot < 2 or rot % 2 or not factor > 0 or not base > 0:
        raise ValueError("rot must be even and positive, base and factor positive")
    n = rot // 2
    p = torch.arange(n, dtype=torch.float64)
    magnitude = 1.0
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-p / n)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if not trained > 0 or not fast > slow:
            raise ValueError("parts needs the trained length, and fast above slow")
        turns = trained * f / (2 * math.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0.0, 1.0)
        f = f / factor * (1.0 - keep) + f * keep
        magnitude = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    elif scaling not in ("none", "base"):
        raise ValueError(f"scaling must be none, linear, base or parts, got {scaling!r}")
    return f.float().to(device), magnitude


def rotate(x, positions, freqs, layout: str = "half", magnitude: float = 1.0, inverse: bool = False, out=None):
    """``x`` [B, L, H, D] with the first 2 * len(freqs) elements of every head turned in pairs by position * freqs[p].

    ``positions``: int32 [B, L], or None (0, 1, ...).  ``layout``: "half" (pair p: elements p and p + rot/2) or
    "interleaved" (2p and 2p + 1).  ``inverse`` turns the other way, which is also the gradient.  ``out`` may be ``x``."""
    done = _calls().rotate(x, positions, freqs, _layout(layout), magnitude, inverse, out)
    if done is None:
        _constant(freqs, "freqs")
        return _function(2).apply(x, positions, freqs, layout, magnitude, inverse)
    rc, out = done
    if rc:
        raise PerError(rc, "per_rotate")
    return out


def norm_rotate(q, k, q_weight, k_weight, positions, freqs, eps: float = 1e-6, layout: str = "half", magnitude: float = 1.0,
                q_out=None, k_out=None):
    """Queries and keys divided by the root of the mean square (plus ``eps``) of each head, times their weights (fp32 [D],
    or None), then turned as by ``rotate``, in one pass.  Returns (q_out, k_out), which may be q and k."""
    done = _calls().norm_rotate(q, k, q_weight, k_weight, positions, freqs, _layout(layout), magnitude, eps, q_out, k_out)
    if done is None:
        return norm_rotate_autograd(q, k, q_weight, k_weight, positions, freqs, eps, layout, magnitude)
    rc, q_out, k_out = done
    if rc:
        raise PerError(rc, "per_norm_rotate")
    return q_out, k_out


def norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, positions, freqs, eps: float = 1e-6, layout: str = "half",
                         magnitude: float = 1.0, dq=None, dk=None, want_weights: bool = True):
    """Gradient of ``norm_rotate``: (dq, dk, dq_weight, dk_weight), the last two None without ``want_weights``.
    dq may be dq_out, dk may be dk_out."""
    rc, dq, dk, dqw, dkw = _calls().norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, positions, freqs, _layout(layout),
                                                         magnitude, eps, dq, dk, want_weights)
    if rc:
        raise PerError(rc, "per_norm_rotate_backward")
    return dq, dk, dqw, dkw


# ------------------------------------------------------------------------------------------------------ linear attention
def linear_attention(q, k, v, log_decay, state=None, lengths=None, scale=None, out=None, out_state=None, want_state: bool = True):
    """S[t] = exp(log_decay[h]) S[t-1] + k[t] v[t]^T;  out[t] = scale q[t]^T S[t].  Returns (out, last state or None).

    q [B, L, H, dk]; k [B, L, G, dk] and v [B, L, G, dv] with G dividing H; ``log_decay`` fp32 [H], at most 0; ``state`` fp32
    [B, H, dk, dv] or None (zeros); ``lengths`` int32 [B] or None: valid tokens of each sequence (behind them nothing is read
    and the outputs are zeros); ``scale``: 1 / sqrt(dk) if None.  In bfloat16 two factors inside are rounded to it, besides the
    outputs (``include/per_seq.h``); states are fp32 sums."""
    done = _calls().linear_attention(q, k, v, log_decay, state, lengths, scale, out, out_state, want_state or out_state is not None)
    if done is None:
        out, last = linear_attention_autograd(q, k, v, log_decay, state, lengths, scale)
        return out, last if want_state else None
    rc, out, last = done
    if rc:
        raise PerError(rc, "per_linear_attention")
    return out, last


def linear_attention_backward(dout, q, k, v, log_decay, state=None, dstate=None, lengths=None, scale=None, dq=None, dk=None, dv=None,
                              dstate0=None, want_dstate: bool = True):
    """Gradient of ``linear_attention`` (the decays are constants): from ``dout`` and ``dstate`` (of the last state; None: zeros) to
    (dq, dk, dv, gradient of ``state`` or None)."""
    rc, dq, dk, dv, first = _calls().linear_attention_backward(dout, q, k, v, log_decay, state, dstate, lengths, scale, dq, dk, dv, dstate0,
                                                               want_dstate or dstate0 is not None)
    if rc:
        raise PerError(rc, "per_linear_attention_backward")
    return dq, dk, dv, first


def linear_attention_step(q, k, v, log_decay, state, active=None, scale=None, out=None):
    """One token (length 1) of ``linear_attention`` with the states [B, H, dk, dv] updated in place.  ``active`` int32 [B] or None:
    where it is 0 the state is not touched and the output is zero.  No gradient is formed: refused where one is asked for.  Returns out."""
    rc, out = _calls().linear_attention_step(q, k, v, log_decay, state, active, scale, out)
    if rc:
        raise PerError(rc, "per_linear_attention_step")
    return out


# ------------------------------------------------------------------------------------------------------------- autograd
def _functions():
    import torch
    from torch.autograd.function import once_differentiable

    class NormRotate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, q_weight, k_weight, positions, freqs, eps, layout, magnitude):
            ctx.save_for_backward(q, k, q_weight, k_weight, positions, freqs)
            ctx.how = (eps, layout, magnitude)
            return norm_rotate(q, k, q_weight, k_weight, positions, freqs, eps, layout, magnitude)

        @staticmethod
        @once_differentiable
        def backward(ctx, dq_out, dk_out):
            q, k, qw, kw, positions, freqs = ctx.saved_tensors
            want = ctx.needs_input_grad[2] or ctx.needs_input_grad[3]
            dq, dk, dqw, dkw = norm_rotate_backward(dq_out.contiguous(), dk_out.contiguous(), q, k, qw, kw, positions, freqs, *ctx.how,
                                                    want_weights=want)
            return dq, dk, dqw if qw is not None else None, dkw if kw is not None else None, None, None, None, None, None

    class LinearAttention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, log_decay, state, lengths, scale):
            ctx.save_for_backward(q, k, v, log_decay, state, lengths)
            ctx.scale = scale
            return linear_attention(q, k, v, log_decay, state, lengths, scale)

        @staticmethod
        @once_differentiable
        def backward(ctx, dout, dstate):
            q, k, v, log_decay, state, lengths = ctx.saved_tensors
            want = ctx.needs_input_grad[4]
            dq, dk, dv, first = linear_attention_backward(dout.contiguous(), q, k, v, log_decay, state, None if dstate is None else dstate.contiguous(),
                                                          lengths, ctx.scale, want_dstate=want)
            return dq, dk, dv, None, first, None, None

    class Rotate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, positions, freqs, layout, magnitude, inverse):
            ctx.save_for_backward(positions, freqs)
            ctx.how = (layout, magnitude, not inverse)
            return rotate(x, positions, freqs, layout, magnitude, inverse)

        @staticmethod
        def backward(ctx, dout):
            return rotate(dout.contiguous(), *ctx.saved_tensors, *ctx.how), None, None, None, None, None

    return NormRotate, LinearAttention, Rotate


_FUNCTIONS = None


def _function(i):
    global _FUNCTIONS
    if _FUNCTIONS is None:
        _FUNCTIONS = _functions()
    return _FUNCTIONS[i]


def _constant(t, name):
    import torch
    if isinstance(t, torch.Tensor) and t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: no gradient of it is formed; detach it")


def norm_rotate_autograd(q, k, q_weight, k_weight, positions, freqs, eps: float = 1e-6, layout: str = "half", magnitude: float = 1.0):
    """``norm_rotate`` as a node of torch's graph: gradients of q, k and the weights, once (``freqs`` are constants)."""
    _constant(freqs, "freqs")
    return _function(0).apply(q, k, q_weight, k_weight, positions, freqs, eps, layout, magnitude)


def linear_attention_autograd(q, k, v, log_decay, state=None, lengths=None, scale=None):
    """``linear_attention`` as a node of torch's graph: gradients of q, k, v and ``state``, once (the decays are constants)."""
    _constant(log_decay, "log_decay")
    return _function(1).apply(q, k, v, log_decay, state, lengths, scale)
