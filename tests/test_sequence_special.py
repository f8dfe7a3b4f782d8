"""The sequence operators on values that are not finite: they reach all that depends on them and nothing else, whichever way a sequence
is computed.  Bounds as in test_sequence.py."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import sequence_oracle as oracle  # noqa: E402
from test_sequence import BF16, F32, absolute, attention_inputs, normal, out_bound, state_bound, within  # noqa: E402
from paper_2311_09445_amd import sequence as seq  # noqa: E402


def lost(got, want):
    """How many of the places that are not finite by the definition are."""
    got = got.detach().cpu()
    return int((got.isfinite() & ~want.isfinite()).sum())


# few rows, computed in segments; many, each computed by one workgroup from end to end
@pytest.mark.parametrize("B,L,H,G,dk,dv", [(1, 2600, 2, 1, 64, 48), (1, 4100, 2, 2, 128, 128), (3, 1001, 2, 1, 17, 90), (300, 200, 2, 2, 32, 32)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")], ids=["nan", "inf"])
def test_values_that_are_not_finite_reach_all_that_depends_on_them(B, L, H, G, dk, dv, dtype, bad):
    """However long ago, and however fast the state decays."""
    q, k, v, g, S, _ = attention_inputs(B, L, H, G, dk, dv, dtype)
    dout, dS = normal(11, B, L, H, dv, dtype=dtype), normal(12, B, H, dk, dv)
    for t, at in ((k, 3), (v, L // 2), (q, L - 2), (dout, L - 70)):
        t[0, at, 0, 1] = bad
    few = [t[:1] for t in (q, k, v)]
    out, last = seq.linear_attention(q, k, v, g, S, scale=0.3)
    for x, want in zip((out, last), oracle.attention(*few, g, S[:1], None, 0.3)):
        assert lost(x[:1], want) == 0
        assert bool(x[1:].isfinite().all())
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, scale=0.3)
    for x, want in zip(got, oracle.attention_backward(dout[:1], *few, g, S[:1], dS[:1], None, 0.3)):
        assert lost(x[:1], want) == 0
        assert bool(x[1:].isfinite().all())


def same_places(got, want, bound, what):
    """Finite where the definition is, and right there."""
    got = got.detach().cpu()
    here = want.isfinite()
    wrong = int((got.isfinite() != here).sum())
    assert wrong == 0, f"{what}: {wrong} places of {here.numel()}"
    within(got[here], want[here], bound[here], what)


# one workgroup to a sequence, several heads to one (few and many heads that share), segments; pieces straight to LDS, through
# registers, and single elements
@pytest.mark.parametrize("B,L,H,G,dk,dv", [
    (5, 75, 2, 2, 64, 64), (5, 70, 2, 1, 128, 128), (5, 40, 2, 2, 32, 32), (5, 100, 2, 1, 48, 80), (5, 45, 2, 2, 17, 5), (5, 33, 2, 1, 127, 33),
    (40, 80, 8, 2, 64, 64), (40, 96, 8, 2, 32, 48), (40, 96, 8, 4, 20, 64), (40, 70, 8, 1, 5, 7), (5, 900, 2, 2, 64, 64), (5, 777, 2, 1, 96, 33)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")], ids=["nan", "inf", "-inf"])
def test_values_that_are_not_finite_reach_nothing_else(B, L, H, G, dk, dv, dtype, bad):
    """One in each of five sequences: a value, a key, a query, an output's gradient, a state and its gradient."""
    q, k, v, g, S, _ = attention_inputs(B, L, H, G, dk, dv, dtype)
    dout, dS = normal(11, B, L, H, dv, dtype=dtype), normal(12, B, H, dk, dv)
    lengths = torch.tensor([L - 3 * (b % 4) for b in range(B)], dtype=torch.int32, device="cuda")
    v[0, L // 2, 0, 1] = k[1, L // 2 + 1, -1, 2] = q[2, L // 3, 1, 0] = dout[3, L // 2 + 2, 0, 3] = bad
    S[4, 1, 3, 2] = dS[4, 0, 1, 4] = bad
    few, n = [t[:5] for t in (q, k, v)], lengths[:5].cpu()
    with_few = [t[:5] for t in (S, dS)]
    out, last = seq.linear_attention(q, k, v, g, S, lengths, scale=0.3)
    want, want_state = oracle.attention(*few, g, with_few[0], n, 0.3)
    A, A_state = oracle.attention(*absolute(*few), g, with_few[0].abs(), n, 0.3)
    same_places(out[:5], want, out_bound(dtype, want, A, dk, L), "out")
    same_places(last[:5], want_state, state_bound(A_state, L), "state")
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths, scale=0.3)
    want = oracle.attention_backward(dout[:5], *few, g, *with_few, n, 0.3)
    A = oracle.attention_backward(*absolute(dout[:5], *few), g, *absolute(*with_few), n, 0.3)
    for name, x, w, a, width in zip(("dq", "dk", "dv"), got, want, A, (dv, dv, dk)):
        same_places(x[:5], w, out_bound(dtype, w, a, width, L), name)
    same_places(got[3][:5], want[3], state_bound(A[3], L), "dstate0")
    for x in (out, last, *got):
        assert bool(x[5:].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot,shift", [(37, 20, 0), (64, 32, 1), (64, 32, 0), (200, 64, 0), (201, 66, 0)])
def test_elements_behind_the_rotated_ones_pass(D, rot, shift, layout, dtype):
    """Whatever they are, bit for bit; widths, pairs and addresses that go in vectors and that do not."""
    B, L, H = 2, 5, 3
    x = normal(1, B * L * H * D + 1, dtype=dtype)[shift:shift + B * L * H * D].view(B, L, H, D)
    for i, value in enumerate((float("inf"), float("-inf"), float("nan"), -0.0, 0.0, torch.finfo(dtype).max)):
        x[..., rot + 2 * i] = value
    f, _ = seq.rotary_frequencies(rot)
    bits = torch.int16 if dtype == BF16 else torch.int32
    for inverse in (False, True):
        y = seq.rotate(x, None, f, layout=layout, magnitude=1.5, inverse=inverse)
        same = y[..., rot:].contiguous().view(bits) == x[..., rot:].contiguous().view(bits)
        assert bool((same | (y[..., rot:].isnan() & x[..., rot:].isnan())).all())
        assert bool(y[..., :rot].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(16, 32), (5, 7)])
def test_keys_and_values_that_no_query_reads_have_a_gradient_of_zero(dk, dv, dtype):
    """No heads of queries at all: the sum over none of them, in tensors of the call's and of the caller's (other strides, too)."""
    B, L, G = 2, 9, 3
    q, k, v = normal(1, B, L, 0, dk, dtype=dtype), normal(2, B, L, G, dk, dtype=dtype), normal(3, B, L, G, dv, dtype=dtype)
    dout, g = normal(4, B, L, 0, dv, dtype=dtype), torch.zeros(0, device="cuda")
    out, last = seq.linear_attention(q, k, v, g)
    assert out.shape == (B, L, 0, dv) and last.shape == (B, 0, dk, dv)
    room = torch.full((B, L, G + 1, dk), 7.0, dtype=dtype, device="cuda")
    given_v = torch.full((B, L, G, dv), 7.0, dtype=dtype, device="cuda")
    dq, gk, gv, first = seq.linear_attention_backward(dout, q, k, v, g, dk=room[:, :, 1:], dv=given_v)
    assert dq.shape == q.shape and first.shape == (B, 0, dk, dv)
    assert not gk.any() and not gv.any() and bool((room[:, :, 0] == 7.0).all())
    dirty = [torch.full_like(t, 7.0) for t in (k, v)]
    del dirty       # (memory that a new tensor may well get)
    for t in seq.linear_attention_backward(dout, q, k, v, g, last, last)[1:3]:
        assert not t.any()
