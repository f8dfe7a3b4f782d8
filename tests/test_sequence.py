"""The sequence operators on the GPU against their definitions in 64 bits (tests/sequence_oracle.py).

Bounds.  u is the unit roundoff of the type (2^-8 for bfloat16), e = 2^-24.  An output of the attention is a sum; A is that sum with
every factor replaced by its absolute value (the same recurrence on absolute inputs).  In bfloat16 the kernels may round the products
x.y, the state a chunk starts from and the output: |error| <= u |out| + 2 u A, and a hundredth for the fp32 arithmetic below it.  In
fp32, sums of dk, of 32 and of the chunks, and decays within 2 e (1 + |exponent|), decay * |exponent| <= 1: |error| <= (dk + 64 + L / 16) e A.
States are fp32 sums whatever the inputs' type: (64 + L / 16) e A.
Norm and rotation: a value is a sum of two products of four factors each, of a sum over the head: u |out| + (D + 32) e A with
A = |c| |a| + |s| |b|; the gradients' sums over tokens and heads: (8 + log2 n) 8 e A.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import sequence_oracle as oracle  # noqa: E402
from sequence_oracle import U_BF16, U_F32  # noqa: E402
from paper_2311_09445_amd import sequence as seq  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def unit(dtype):
    return U_BF16 if dtype == BF16 else U_F32


def normal(seed, *shape, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def within(got, want, bound, what):
    got, bound = got.detach().double().cpu(), bound + 1e-30
    off = (got - want).abs()
    bad = ~(off <= bound)
    if bad.any():
        at = tuple(int(i[0]) for i in torch.nonzero(bad, as_tuple=True))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; first at {at}: got {got[at]}, want {want[at]}, bound {bound[at]}")


def absolute(*ts):
    return [None if t is None else t.abs() for t in ts]


def out_bound(dtype, want, A, width, L):
    if dtype == BF16:
        return 1.01 * U_BF16 * (want.abs() + 2 * A)
    return (width + 64 + L / 16) * U_F32 * A


def state_bound(A, L):
    return (64 + L / 16) * U_F32 * A


def decays(H, fast=1.0, slow=2 ** -8):
    return -torch.logspace(math.log2(fast), math.log2(slow), H, base=2).float().cuda()


def attention_inputs(B, L, H, G, dk, dv, dtype, seed=1, ragged=False, state=True):
    q, k, v = normal(seed, B, L, H, dk, dtype=dtype), normal(seed + 1, B, L, G, dk, dtype=dtype), normal(seed + 2, B, L, G, dv, dtype=dtype)
    S = normal(seed + 3, B, H, dk, dv) if state else None
    lengths = None
    if ragged:
        lengths = torch.tensor([(L * (i + 1) * 7) // 11 % (L + 1) for i in range(B)], dtype=torch.int32)
        lengths[0] = L
        if B > 1:
            lengths[1] = 0
        lengths = lengths.cuda()
    return q, k, v, decays(H), S, lengths


def check_attention(q, k, v, g, S, lengths, scale, out, last):
    L, dk = q.shape[1], q.shape[3]
    host = None if lengths is None else lengths.cpu()
    want, want_state = oracle.attention(q, k, v, g, S, host, scale)
    A, A_state = oracle.attention(*absolute(q, k, v), g, *absolute(S), host, abs(scale))
    within(out, want, out_bound(q.dtype, want, A, dk, L), "out")
    if last is not None:
        within(last, want_state, state_bound(A_state, L), "state")


SHAPES = [  # B, L, H, G, dk, dv
    (1, 1, 1, 1, 1, 1), (2, 2, 2, 2, 16, 16), (2, 31, 2, 1, 32, 32), (1, 32, 2, 2, 64, 64), (2, 33, 3, 3, 64, 32),
    (1, 65, 4, 2, 128, 128), (3, 100, 4, 1, 48, 80), (2, 77, 2, 2, 17, 5), (1, 300, 2, 2, 128, 64), (2, 257, 2, 1, 96, 128),
    (1, 64, 1, 1, 8, 128), (1, 50, 2, 2, 127, 33),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,L,H,G,dk,dv", SHAPES)
def test_attention(B, L, H, G, dk, dv, ragged, dtype):
    q, k, v, g, S, lengths = attention_inputs(B, L, H, G, dk, dv, dtype, ragged=ragged)
    out, last = seq.linear_attention(q, k, v, g, S, lengths, scale=0.3)
    check_attention(q, k, v, g, S, lengths, 0.3, out, last)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,L,H,G,dk,dv", SHAPES)
def test_attention_backward(B, L, H, G, dk, dv, ragged, dtype):
    q, k, v, g, S, lengths = attention_inputs(B, L, H, G, dk, dv, dtype, ragged=ragged)
    dout, dS = normal(11, B, L, H, dv, dtype=dtype), normal(12, B, H, dk, dv)
    scale = 0.3
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths, scale=scale)
    host = None if lengths is None else lengths.cpu()
    want = oracle.attention_backward(dout, q, k, v, g, S, dS, host, scale)
    A = oracle.attention_backward(*absolute(dout, q, k, v), g, *absolute(S, dS), host, scale)
    for name, x, w, a, width in zip(("dq", "dk", "dv"), got, want, A, (dv, dv, dk)):
        within(x, w, out_bound(dtype, w, a, width, L), name)
    within(got[3], want[3], state_bound(A[3], L), "dstate0")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_long_axis_few_rows(dtype):
    """Long enough to be cut into pieces that are computed apart and joined."""
    B, L, H, G, dk, dv = 1, 5003, 2, 1, 64, 48
    q, k, v, g, S, _ = attention_inputs(B, L, H, G, dk, dv, dtype)
    g = torch.tensor([-0.5, -2.0 ** -10], device="cuda")
    out, last = seq.linear_attention(q, k, v, g, S, scale=0.125)
    check_attention(q, k, v, g, S, None, 0.125, out, last)
    dout, dS = normal(11, B, L, H, dv, dtype=dtype), normal(12, B, H, dk, dv)
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, None, scale=0.125)
    want = oracle.attention_backward(dout, q, k, v, g, S, dS, None, 0.125)
    A = oracle.attention_backward(*absolute(dout, q, k, v), g, *absolute(S, dS), None, 0.125)
    for name, x, w, a, width in zip(("dq", "dk", "dv"), got, want, A, (dv, dv, dk)):
        within(x, w, out_bound(dtype, w, a, width, L), name)
    within(got[3], want[3], state_bound(A[3], L), "dstate0")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_ragged_long_sequences(dtype):
    B, L, H, G, dk, dv = 5, 2600, 1, 1, 32, 64
    q, k, v, g, S, _ = attention_inputs(B, L, H, G, dk, dv, dtype)
    g = torch.tensor([-0.01], device="cuda")
    lengths = torch.tensor([2600, 0, 1, 513, 2049], dtype=torch.int32, device="cuda")
    out, last = seq.linear_attention(q, k, v, g, S, lengths, scale=0.2)
    check_attention(q, k, v, g, S, lengths, 0.2, out, last)
    dout, dS = normal(11, B, L, H, dv, dtype=dtype), normal(12, B, H, dk, dv)
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths, scale=0.2)
    want = oracle.attention_backward(dout, q, k, v, g, S, dS, lengths.cpu(), 0.2)
    A = oracle.attention_backward(*absolute(dout, q, k, v), g, *absolute(S, dS), lengths.cpu(), 0.2)
    for name, x, w, a, width in zip(("dq", "dk", "dv"), got, want, A, (dv, dv, dk)):
        within(x, w, out_bound(dtype, w, a, width, L), name)
    within(got[3], want[3], state_bound(A[3], L), "dstate0")


def test_gradient_against_differences():
    """The gradient of a weighted sum of outputs and last states against central differences of the oracle's forward in 64 bits."""
    B, L, H, G, dk, dv = 2, 37, 2, 1, 6, 7
    q, k, v, g, S, lengths = attention_inputs(B, L, H, G, dk, dv, F32, ragged=False)
    lengths = torch.tensor([37, 20], dtype=torch.int32, device="cuda")
    dout, dS = normal(11, B, L, H, dv), normal(12, B, H, dk, dv)
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths, scale=0.4)
    A = oracle.attention_backward(*absolute(dout, q, k, v), g, *absolute(S, dS), lengths.cpu(), 0.4)
    rng = np.random.default_rng(3)
    names = ("q", "k", "v", "S")
    for i, (name, grad) in enumerate(zip(names, got)):
        for _ in range(4):
            at = tuple(int(rng.integers(n)) for n in grad.shape)
            value = []
            for sign in (1.0, -1.0):   # (the loss is linear in each single value: the difference is exact but for rounding)
                args = {n: t.detach().cpu().double().clone() for n, t in zip(names, (q, k, v, S))}
                args[name][at] += sign * 0.5
                o, last = oracle.attention(args["q"], args["k"], args["v"], g, args["S"], lengths.cpu(), 0.4)
                value.append(float((o * dout.cpu().double()).sum() + (last * dS.cpu().double()).sum()))
            bound = (dk + 64 + L / 16) * U_F32 * float(A[i][at]) + 1e-10
            assert abs(float(grad[at]) - (value[0] - value[1])) <= bound, (name, at)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_what_lies_behind_the_length_is_not_read(dtype):
    B, L, H, dk, dv = 3, 70, 2, 64, 64
    q, k, v, g, S, _ = attention_inputs(B, L, H, H, dk, dv, dtype)
    dout, dS = normal(11, B, L, H, dv, dtype=dtype), normal(12, B, H, dk, dv)
    lengths = torch.tensor([40, 0, 33], dtype=torch.int32, device="cuda")
    clean = seq.linear_attention(q, k, v, g, S, lengths), seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        for t in (q, k, v, dout):
            for b, n in enumerate(lengths.tolist()):
                t[b, n:] = bad
        again = seq.linear_attention(q, k, v, g, S, lengths), seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)
        for one, two in zip(clean, again):
            for x, y in zip(one, two):
                assert torch.equal(x, y)
    out, last = clean[0]
    for b, n in enumerate(lengths.tolist()):
        assert not out[b, n:].any()
        for x in clean[1][:3]:
            assert not x[b, n:].any()
    assert torch.equal(last[1], S[1]) and torch.equal(clean[1][3][1], dS[1])


def test_lengths_outside_the_range_are_taken_as_its_ends():
    q, k, v, g, S, _ = attention_inputs(3, 20, 2, 2, 16, 16, F32)
    wild = torch.tensor([-5, 1000, 7], dtype=torch.int32, device="cuda")
    tame = torch.tensor([0, 20, 7], dtype=torch.int32, device="cuda")
    for x, y in zip(seq.linear_attention(q, k, v, g, S, wild), seq.linear_attention(q, k, v, g, S, tame)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_decay_at_its_ends(dtype):
    """Keeping nothing (-infinity), keeping everything (0), and decays that leave the range of fp32 within a chunk."""
    B, L, dk, dv = 1, 75, 32, 32
    g = torch.tensor([-math.inf, 0.0, -20.0], device="cuda")
    q, k, v, _, S, _ = attention_inputs(B, L, 3, 3, dk, dv, dtype)
    out, last = seq.linear_attention(q, k, v, g, S, scale=1.0)
    check_attention(q, k, v, g, S, None, 1.0, out, last)
    dout, dS = normal(11, B, L, 3, dv, dtype=dtype), normal(12, B, 3, dk, dv)
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, scale=1.0)
    want = oracle.attention_backward(dout, q, k, v, g, S, dS, None, 1.0)
    A = oracle.attention_backward(*absolute(dout, q, k, v), g, *absolute(S, dS), None, 1.0)
    for name, x, w, a, width in zip(("dq", "dk", "dv"), got, want, A, (dv, dv, dk)):
        within(x, w, out_bound(dtype, w, a, width, L), name)
    within(got[3], want[3], state_bound(A[3], L), "dstate0")


def test_empty_sizes():
    for B, L, H in ((0, 5, 2), (2, 0, 2), (2, 5, 0)):
        q, k, v = (torch.zeros(B, L, H, 16, device="cuda") for _ in range(3))
        g, S = torch.full((H,), -0.1, device="cuda"), normal(1, B, H, 16, 16)
        out, last = seq.linear_attention(q, k, v, g, S)
        assert out.shape == (B, L, H, 16) and torch.equal(last, S)
        dq, dk, dv, dS0 = seq.linear_attention_backward(out, q, k, v, g, S, S)
        assert dq.shape == q.shape and torch.equal(dS0, S)
        x = seq.rotate(q, None, torch.ones(8, device="cuda"))
        assert x.shape == q.shape
        a, b = seq.norm_rotate(q, k, None, None, None, torch.ones(8, device="cuda"))
        assert a.shape == q.shape and b.shape == k.shape
        w = torch.ones(16, device="cuda")
        back = seq.norm_rotate_backward(q, k, q, k, w, w, None, torch.ones(8, device="cuda"))
        assert not back[2].any() and not back[3].any()


def test_without_state_and_in_place_state():
    q, k, v, g, S, lengths = attention_inputs(3, 45, 2, 2, 32, 64, BF16, ragged=True)
    zero = torch.zeros_like(S)
    a, b = seq.linear_attention(q, k, v, g, None, lengths), seq.linear_attention(q, k, v, g, zero, lengths)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out, none = seq.linear_attention(q, k, v, g, S, lengths, want_state=False)
    out2, last = seq.linear_attention(q, k, v, g, S, lengths)
    assert none is None and out.shape == out2.shape
    T = S.clone()
    _, same = seq.linear_attention(q, k, v, g, T, lengths, out_state=T)
    assert same is T and torch.equal(T, last)
    dout, dS = normal(11, 3, 45, 2, 64, dtype=BF16), normal(12, *S.shape)
    want = seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)
    D = dS.clone()
    got = seq.linear_attention_backward(dout, q, k, v, g, S, D, lengths, dstate0=D)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_strided_views(dtype):
    """Queries, keys and values side by side in one tensor, heads before tokens, sizes and offsets that break the alignment,
    a key shared by the whole batch."""
    B, L, H, d = 2, 41, 4, 32
    packed = normal(5, B, L, 3 * H * d + 3, dtype=dtype)
    q, k, v = (packed[..., 1 + i * H * d:1 + (i + 1) * H * d].unflatten(-1, (H, d)) for i in range(3))
    g, S = decays(H), normal(6, B, H, d, d)
    want = seq.linear_attention(*(t.contiguous() for t in (q, k, v)), g, S)
    out = torch.empty(B, H, L, d, dtype=dtype, device="cuda").transpose(1, 2)
    got = seq.linear_attention(q, k, v, g, S, out=out)
    assert got[0] is out or got[0].data_ptr() == out.data_ptr()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = k[:1].contiguous()
    shared = one.expand(B, L, H, d)
    x, y = seq.linear_attention(q, shared, v, g, S), seq.linear_attention(q.contiguous(), shared.contiguous(), v.contiguous(), g, S)
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    dout = normal(7, B, H, L, d, dtype=dtype).transpose(1, 2)
    x = seq.linear_attention_backward(dout, q, shared, v, g, S)
    y = seq.linear_attention_backward(dout.contiguous(), q.contiguous(), shared.contiguous(), v.contiguous(), g, S)
    for a, b in zip(x, y):
        assert torch.equal(a, b)


def test_results_do_not_change_from_call_to_call():
    q, k, v, g, S, lengths = attention_inputs(4, 700, 4, 2, 64, 64, BF16, ragged=True)
    dout, dS = normal(11, 4, 700, 4, 64, dtype=BF16), normal(12, *S.shape)
    first = [*seq.linear_attention(q, k, v, g, S, lengths), *seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)]
    for _ in range(3):
        again = [*seq.linear_attention(q, k, v, g, S, lengths), *seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)]
        for x, y in zip(first, again):
            assert torch.equal(x, y)


# --------------------------------------------------------------------------------------------------------------- one token
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,dk,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 64, 64), (2, 2, 2, 128, 128), (5, 3, 1, 48, 80), (2, 2, 2, 17, 5), (70, 4, 4, 32, 128),
                                         (2, 1, 1, 127, 33), (3, 2, 2, 100, 126)])
def test_step(B, H, G, dk, dv, dtype):
    q, k, v, g, S, _ = attention_inputs(B, 1, H, G, dk, dv, dtype)
    active = torch.tensor([i % 3 != 1 for i in range(B)], dtype=torch.int32, device="cuda")
    for act in (None, active):
        T = S.clone()
        out = seq.linear_attention_step(q, k, v, g, T, act, scale=0.3)
        want, want_state = oracle.attention(q, k, v, g, S, None if act is None else act.cpu(), 0.3)
        A, A_state = oracle.attention(*absolute(q, k, v), g, S.abs(), None if act is None else act.cpu(), 0.3)
        within(out, want, unit(dtype) * want.abs() + (dk + 32) * U_F32 * A, "out")
        within(T, want_state, 8 * U_F32 * A_state, "state")
        if act is not None and B > 1:
            assert torch.equal(T[1], S[1]) and not out[1].any()


def test_steps_follow_the_sequence():
    B, L, H, d = 2, 40, 2, 64
    q, k, v, g, S, _ = attention_inputs(B, L, H, H, d, d, F32)
    T = S.clone()
    outs = [seq.linear_attention_step(*(t[:, i:i + 1] for t in (q, k, v)), g, T) for i in range(L)]
    check_attention(q, k, v, g, S, None, d ** -0.5, torch.cat(outs, 1), T)


def test_states_in_a_larger_pool():
    """States that are a slice of a pool with other strides; the rest of the pool stays as it is."""
    B, H, d = 3, 2, 32
    q, k, v, g, _, _ = attention_inputs(B, 1, H, H, d, d, BF16)
    pool = normal(9, 2 * B, H + 1, d, d)
    before = pool.clone()
    view = pool[::2, :H]
    want = view.clone()
    a = seq.linear_attention_step(q, k, v, g, view)
    b = seq.linear_attention_step(q, k, v, g, want)
    assert torch.equal(a, b) and torch.equal(view, want)
    assert torch.equal(pool[1::2], before[1::2]) and torch.equal(pool[:, H:], before[:, H:])


# ------------------------------------------------------------------------------------------------------ rotation and norms
ROTARY = [  # B, L, H, G, D, rot
    (1, 1, 1, 1, 2, 2), (2, 3, 2, 1, 64, 64), (1, 5, 4, 2, 128, 128), (2, 7, 3, 1, 128, 64), (1, 4, 2, 2, 80, 40), (1, 3, 5, 5, 33, 20),
    (1, 9, 8, 2, 96, 48), (2, 2, 1, 1, 256, 256), (1, 3, 2, 1, 16, 0), (1, 2, 2, 2, 7, 6), (1, 2, 33, 3, 32, 32), (3, 1, 2, 2, 240, 176), (1, 67, 4, 4, 64, 32),
]


def rotary_inputs(B, L, H, G, D, rot, dtype, far):
    q, k = normal(1, B, L, H, D, dtype=dtype), normal(2, B, L, G, D, dtype=dtype)
    wq, wk = 1 + 0.2 * normal(3, D), 1 + 0.2 * normal(4, D)
    pos = (torch.arange(B)[:, None] * 977 + torch.arange(L) + far).int().cuda()
    if rot:
        f, m = seq.rotary_frequencies(rot, scaling="linear", factor=4.0)
    else:
        f, m = torch.empty(0, device="cuda"), 1.0
    return q, k, wq, wk, pos, f, 1.1


def spread(x, positions, f, layout, magnitude, inverse=False):
    """|c| |a| + |s| |b| of every element: at most the magnitude times the sum of the pair's absolute values."""
    rot = 2 * len(f)
    y = oracle.f64(x).abs().clone()
    if layout == "half":
        both = y[..., :rot // 2] + y[..., rot // 2:rot]
        y[..., :rot] = magnitude * torch.cat((both, both), -1)
    else:
        both = y[..., 0:rot:2] + y[..., 1:rot:2]
        y[..., :rot] = magnitude * both.repeat_interleave(2, -1)
    return y


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("far", [0, 1 << 20, -3])
@pytest.mark.parametrize("B,L,H,G,D,rot", ROTARY)
def test_rotate(B, L, H, G, D, rot, far, layout, dtype):
    q, _, _, _, pos, f, m = rotary_inputs(B, L, H, G, D, rot, dtype, far)
    for inverse in (False, True):
        got = seq.rotate(q, pos, f, layout, m, inverse)
        want = oracle.turned(q, pos.cpu(), f.cpu(), layout, m, inverse)
        within(got, want, unit(dtype) * want.abs() + 32 * U_F32 * spread(q, pos, f, layout, m), "rotated")
    assert torch.equal(got[..., rot:], q[..., rot:])
    x = q.clone()
    assert torch.equal(seq.rotate(x, pos, f, layout, m, True, out=x), got)
    if far == 0 and B == 1:
        assert torch.equal(seq.rotate(q, None, f, layout, m), seq.rotate(q, pos, f, layout, m))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("B,L,H,G,D,rot", ROTARY)
def test_norm_rotate(B, L, H, G, D, rot, weights, layout, dtype):
    q, k, wq, wk, pos, f, m = rotary_inputs(B, L, H, G, D, rot, dtype, 5000)
    if not weights:
        wq = wk = None
    got = seq.norm_rotate(q, k, wq, wk, pos, f, 1e-5, layout, m)
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        want = oracle.norm_rotate(x, w, pos.cpu(), f.cpu(), 1e-5, layout, m)
        A = spread(oracle.normed(x, w, 1e-5), pos, f, layout, m)
        within(y, want, unit(dtype) * want.abs() + (D + 32) * U_F32 * A, "normed and rotated")
    a, b = q.clone(), k.clone()
    seq.norm_rotate(a, b, wq, wk, pos, f, 1e-5, layout, m, q_out=a, k_out=b)
    assert torch.equal(a, got[0]) and torch.equal(b, got[1])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("B,L,H,G,D,rot", ROTARY)
def test_norm_rotate_backward(B, L, H, G, D, rot, weights, layout, dtype):
    q, k, wq, wk, pos, f, m = rotary_inputs(B, L, H, G, D, rot, dtype, 5000)
    if not weights:
        wq = wk = None
    gq, gk = normal(7, B, L, H, D, dtype=dtype), normal(8, B, L, G, D, dtype=dtype)
    got = seq.norm_rotate_backward(gq, gk, q, k, wq, wk, pos, f, 1e-5, layout, m)
    for x, w, d, dx, dw in ((q, wq, gq, got[0], got[2]), (k, wk, gk, got[1], got[3])):
        want, want_w = oracle.norm_rotate_backward(d, x, w, pos.cpu(), f.cpu(), 1e-5, layout, m)
        dy = spread(d, pos, f, layout, m)
        h = dy if w is None else dy * oracle.f64(w).abs()
        xa = oracle.f64(x).abs()
        root = (xa.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt()
        A = h / root + xa * (h * xa).sum(-1, keepdim=True) / (D * root ** 3)
        within(dx, want, unit(dtype) * want.abs() + (2 * D + 32) * U_F32 * A, "gradient of rows")
        n = x.numel() // D
        within(dw, want_w, (D + 32 + n) * U_F32 * (dy * xa / root).sum((0, 1, 2)), "gradient of weight")
    again = seq.norm_rotate_backward(gq, gk, q, k, wq, wk, pos, f, 1e-5, layout, m)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    a, b = gq.clone(), gk.clone()
    dq, dk, none, none2 = seq.norm_rotate_backward(a, b, q, k, wq, wk, pos, f, 1e-5, layout, m, dq=a, dk=b, want_weights=False)
    assert none is None and none2 is None and torch.equal(a, got[0]) and torch.equal(b, got[1])


def test_norm_gradient_against_differences():
    B, L, H, G, D, rot = 1, 3, 2, 1, 12, 8
    q, k, wq, wk, pos, f, m = rotary_inputs(B, L, H, G, D, rot, F32, 100)
    gq, gk = normal(7, B, L, H, D), normal(8, B, L, G, D)
    dq, _, dwq, _ = seq.norm_rotate_backward(gq, gk, q, k, wq, wk, pos, f, 1e-5, "half", m)

    def loss(x, w):
        return float((oracle.norm_rotate(x, w, pos.cpu(), f.cpu(), 1e-5, "half", m) * oracle.f64(gq)).sum())

    rng = np.random.default_rng(5)
    x0, w0, d = oracle.f64(q), oracle.f64(wq), 1e-5
    for _ in range(6):
        at = tuple(int(rng.integers(n)) for n in q.shape)
        x1, x2 = x0.clone(), x0.clone()
        x1[at] += d
        x2[at] -= d
        # a central difference is off by d^2 times a third derivative (of order 10 here), and the kernel by fp32 sums of order 10
        assert abs(float(dq[at]) - (loss(x1, w0) - loss(x2, w0)) / (2 * d)) <= 1e-4
        e = at[-1]
        w1, w2 = w0.clone(), w0.clone()
        w1[e] += d
        w2[e] -= d
        assert abs(float(dwq[e]) - (loss(x0, w1) - loss(x0, w2)) / (2 * d)) <= 1e-4


def test_a_head_of_zeros_stays_zero():
    q = torch.zeros(1, 2, 2, 64, device="cuda", dtype=BF16)
    f, _ = seq.rotary_frequencies(64)
    a, b = seq.norm_rotate(q, q.clone(), None, None, None, f)
    assert not a.any() and not b.any()
    d = normal(1, 1, 2, 2, 64, dtype=BF16)
    dq, _, _, _ = seq.norm_rotate_backward(d, d.clone(), q, q.clone(), None, None, None, f)
    want, _ = oracle.norm_rotate_backward(d, q, None, None, f.cpu(), 1e-6, "half", 1.0)
    within(dq, want, U_BF16 * want.abs() + 100 * U_F32 * 1e3 * spread(d, None, f, "half", 1.0), "gradient at zero")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_strided_views(layout, dtype):
    B, L, H, D = 2, 11, 4, 64
    packed = normal(5, B, L, 2 * H * D + 5, dtype=dtype)
    f, _ = seq.rotary_frequencies(D)
    for offset in (0, 1, 4):
        q, k = (packed[..., offset + i * H * D:offset + (i + 1) * H * D].unflatten(-1, (H, D)) for i in range(2))
        pos = torch.arange(100, 100 + L, dtype=torch.int32, device="cuda").expand(B, L)
        wq = 1 + 0.1 * normal(3, D)
        # the same values through another access width: only the order of a head's sum of squares may differ
        want = oracle.norm_rotate(q, wq, pos.cpu(), f.cpu(), 1e-6, layout, 1.0)
        got = seq.norm_rotate(q, k, wq, wq, pos, f, layout=layout)
        A = spread(oracle.normed(q, wq, 1e-6), pos, f, layout, 1.0)
        within(got[0], want, unit(dtype) * want.abs() + (D + 32) * U_F32 * A, "strided")
        out = torch.empty(B, H, L, D, dtype=dtype, device="cuda").transpose(1, 2)
        seq.rotate(q, pos, f, layout, out=out)
        want = oracle.turned(q, pos.cpu(), f.cpu(), layout, 1.0)
        within(out, want, unit(dtype) * want.abs() + 32 * U_F32 * spread(q, pos, f, layout, 1.0), "strided rotation")


# ------------------------------------------------------------------------------------------------------- streams and graphs
def test_on_a_stream_of_its_own():
    q, k, v, g, S, lengths = attention_inputs(3, 1500, 2, 2, 64, 64, BF16, ragged=True)
    dout, dS = normal(11, 3, 1500, 2, 64, dtype=BF16), normal(12, *S.shape)
    want = [*seq.linear_attention(q, k, v, g, S, lengths), *seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [*seq.linear_attention(q, k, v, g, S, lengths), *seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths)]
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_in_a_graph():
    B, L, H, d = 2, 600, 2, 64
    q, k, v, g, S, _ = attention_inputs(B, L, H, H, d, d, BF16)
    f, _ = seq.rotary_frequencies(d)
    w = torch.ones(d, device="cuda")
    dout = normal(11, B, L, H, d, dtype=BF16)
    T = S.clone()

    def work(T):
        a, b = seq.norm_rotate(q, k, w, w, None, f)
        out, last = seq.linear_attention(a, b, v, g, S)
        da, db, dv, _ = seq.linear_attention_backward(dout, a, b, v, g, S)
        back = seq.norm_rotate_backward(da, db, q, k, w, w, None, f)
        step = seq.linear_attention_step(q[:, :1], k[:, :1], v[:, :1], g, T)
        return [out, last, dv, *back, step]

    work(T)
    torch.cuda.synchronize()
    T.copy_(S)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(T)
    E = S.clone()
    for i in range(4):
        q.copy_(normal(20 + i, *q.shape, dtype=BF16))
        dout.copy_(normal(40 + i, *dout.shape, dtype=BF16))
        graph.replay()
        want = work(E)          # (eager work between the replays)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), f"replay {i}"
        assert torch.equal(T, E)


def test_autograd():
    B, L, H, G, d = 2, 50, 4, 2, 32
    q, k, v, g, S, lengths = attention_inputs(B, L, H, G, d, d, F32, ragged=True)
    w = 1 + 0.1 * normal(9, d)
    f, _ = seq.rotary_frequencies(d)
    leaves = [t.clone().requires_grad_() for t in (q, k, v, S, w)]
    a, b = seq.norm_rotate_autograd(leaves[0], leaves[1], leaves[4], None, None, f)
    out, last = seq.linear_attention_autograd(a, b, leaves[2], g, leaves[3], lengths)
    dout, dS = normal(11, *out.shape), normal(12, *last.shape)
    torch.autograd.backward((out, last), (dout, dS))
    a, b = seq.norm_rotate(q, k, w, None, None, f)
    da, db, dv, dS0 = seq.linear_attention_backward(dout, a, b, v, g, S, dS, lengths)
    dq, dk, dw, _ = seq.norm_rotate_backward(da, db, q, k, w, None, None, f)
    for t, want in zip(leaves, (dq, dk, dv, dS0, dw)):
        assert torch.equal(t.grad, want)


# ---------------------------------------------------------------------------------------------------------------- refusals
def test_refusals():
    q, k, v, g, S, _ = attention_inputs(2, 8, 4, 2, 16, 16, BF16)
    f, _ = seq.rotary_frequencies(16)
    refused = [
        lambda: seq.linear_attention(q.half(), k.half(), v.half(), g),
        lambda: seq.linear_attention(q, k.float(), v, g),
        lambda: seq.linear_attention(q, k[:, :4], v, g),
        lambda: seq.linear_attention(q[:, :, :3], k, v, g[:3]),
        lambda: seq.linear_attention(q, k, v, g[:2]),
        lambda: seq.linear_attention(q, k, v, g.double()),
        lambda: seq.linear_attention(q, k, v, g, S[:1]),
        lambda: seq.linear_attention(q, k, v, g, S.transpose(2, 3)),
        lambda: seq.linear_attention(q, k, v, g, S, torch.ones(2, dtype=torch.int64, device="cuda")),
        lambda: seq.linear_attention(q, k, v, g, S, torch.ones(3, dtype=torch.int32, device="cuda")),
        lambda: seq.linear_attention(q.transpose(2, 3).contiguous().transpose(2, 3), k, v, g),
        lambda: seq.linear_attention(q.cpu(), k, v, g),
        lambda: seq.linear_attention(q, k.cpu(), v, g),
        lambda: seq.linear_attention(q, k, v, g, out=q.float()),
        lambda: seq.linear_attention_step(q, k, v, g, None),
        lambda: seq.linear_attention_backward(None, q, k, v, g),
        lambda: seq.linear_attention_backward(q[:, :, :2], q, k, v, g),
        lambda: seq.rotate(q[0], None, f),
        lambda: seq.rotate(q, torch.zeros(2, 8, dtype=torch.int64, device="cuda"), f),
        lambda: seq.rotate(q, None, torch.ones(9, device="cuda")),
        lambda: seq.rotate(q, None, f, layout="both"),
        lambda: seq.norm_rotate(q, k, torch.ones(8, device="cuda"), None, None, f),
        lambda: seq.norm_rotate(q, k[..., :8], None, None, None, f),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((ValueError, TypeError)):
            call()
            print("not refused:", i)
    out_of_range = [
        lambda: seq.linear_attention_step(q, k, v, g, S),                              # more than one token
        lambda: seq.linear_attention(*(torch.zeros(1, 2, 1, 129, device="cuda") for _ in range(3)), g[:1]),
        lambda: seq.linear_attention(q, q, v.expand(2, 8, 2, 16).repeat(1, 1, 2, 1), g, out=q),   # out is an input
        lambda: seq.linear_attention(q, k, v, g, S, out=torch.empty(2, 8, 1, 16, dtype=BF16, device="cuda").expand(2, 8, 4, 16)),
        lambda: seq.linear_attention_backward(q, q, k, v, g, S, S, dstate0=S),         # the gradient over the state
        lambda: seq.linear_attention(q, k, v, g, scale=float("nan")),
        lambda: seq.rotate(torch.zeros(1, 1, 1, 257, device="cuda"), None, f),
        lambda: seq.norm_rotate(q, k, None, None, None, f, eps=-1.0),
        lambda: seq.rotate(q, None, f, magnitude=float("inf")),
    ]
    for call in out_of_range:
        with pytest.raises(seq.PerError):
            call()
    torch.cuda.synchronize()
