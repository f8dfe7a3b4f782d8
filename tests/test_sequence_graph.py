"""The sequence operators in torch's graph: nothing is lost from a gradient without an error."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_sequence import BF16, F32, attention_inputs, normal  # noqa: E402
from paper_2311_09445_amd import sequence as seq  # noqa: E402


def leaves(*ts):
    return [t.clone().requires_grad_() for t in ts]


def test_no_second_derivatives():
    """A gradient of a gradient through an operator is refused; without its part it would be a wrong one."""
    q, k, v, g, S, _ = attention_inputs(2, 20, 2, 2, 16, 16, F32)
    f, _ = seq.rotary_frequencies(16)
    w = torch.ones(16, device="cuda")
    for call in (lambda q, k: seq.linear_attention_autograd(q, k, v, g, S)[0], lambda q, k: seq.norm_rotate_autograd(q, k, w, None, None, f)[0]):
        a, b = leaves(q, k)
        loss = call(a, b).square().sum() + a.pow(3).sum()
        first, = torch.autograd.grad(loss, a, create_graph=True)
        with pytest.raises(RuntimeError):
            first.square().sum().backward()


def test_constants_that_ask_for_a_gradient_are_refused():
    """No gradient of decays and frequencies is formed: None for it would be a wrong one."""
    q, k, v, g, S, _ = attention_inputs(2, 20, 2, 2, 16, 16, F32)
    f, _ = seq.rotary_frequencies(16)
    asked_g, asked_f = leaves(g, f)
    a, b = leaves(q, k)
    with pytest.raises(ValueError, match="log_decay"):
        seq.linear_attention_autograd(a, b, v, asked_g, S)
    with pytest.raises(ValueError, match="freqs"):
        seq.norm_rotate_autograd(a, b, None, None, None, asked_f)
    with torch.no_grad():       # nothing is asked for here
        out, _ = seq.linear_attention_autograd(a, b, v, asked_g, S)
        x, _ = seq.norm_rotate_autograd(a, b, None, None, None, asked_f)
    assert torch.equal(out, seq.linear_attention_autograd(q, k, v, g, S)[0]) and torch.equal(x, seq.norm_rotate_autograd(q, k, None, None, None, f)[0])
    assert not out.requires_grad and not x.requires_grad


def test_tensors_written_in_place_are_noticed():
    """Torch's check of what it has kept for a gradient sees every tensor of the caller's that a call writes."""
    q, k, v, g, S, _ = attention_inputs(2, 1, 2, 2, 16, 16, F32)
    f, _ = seq.rotary_frequencies(16)
    dout, dS = normal(11, *q.shape), normal(12, *S.shape)
    room = torch.empty_like
    writes = {
        "step": (lambda: S, lambda t: seq.linear_attention_step(q, k, v, g, t)),
        "step's out": (lambda: q, lambda t: seq.linear_attention_step(k, k, v, g, S.clone(), out=t)),
        "out": (lambda: q, lambda t: seq.linear_attention(k, k, v, g, S, out=t)),
        "out_state": (lambda: S, lambda t: seq.linear_attention(q, k, v, g, t, out_state=t)),
        "dq": (lambda: q, lambda t: seq.linear_attention_backward(dout, k, k, v, g, S, dS, dq=t)),
        "dk": (lambda: q, lambda t: seq.linear_attention_backward(dout, k, k, v, g, S, dS, dk=t)),
        "dv": (lambda: q, lambda t: seq.linear_attention_backward(dout, k, k, v, g, S, dS, dv=t)),
        "dstate0": (lambda: S, lambda t: seq.linear_attention_backward(dout, q, k, v, g, None, dS, dstate0=t)),
        "rotate": (lambda: q, lambda t: seq.rotate(t, None, f, out=t)),
        "q_out": (lambda: q, lambda t: seq.norm_rotate(t, k, None, None, None, f, q_out=t)),
        "k_out": (lambda: q, lambda t: seq.norm_rotate(k, t, None, None, None, f, k_out=t)),
        "norm's dq": (lambda: q, lambda t: seq.norm_rotate_backward(dout, dout, k, k, None, None, None, f, dq=t)),
        "norm's dk": (lambda: q, lambda t: seq.norm_rotate_backward(dout, dout, k, k, None, None, None, f, dk=t)),
    }
    for name, (make, write) in writes.items():
        kept = make().clone()
        x, = leaves(room(kept).fill_(2.0))
        loss = (x * kept).sum()
        write(kept)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
            print("not noticed:", name)
    T = S.clone()
    a, b = leaves(q, k)
    out, _ = seq.linear_attention_autograd(a, b, v, g, T)
    seq.linear_attention_step(q, k, v, g, T)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_what_is_only_read_stays_as_it_is_for_the_graph():
    q, k, v, g, S, _ = attention_inputs(2, 9, 2, 2, 16, 16, BF16)
    f, _ = seq.rotary_frequencies(16)
    before = [t._version for t in (q, k, v, g, S, f)]
    out, last = seq.linear_attention(q, k, v, g, S)
    seq.linear_attention_backward(out, q, k, v, g, S, last)
    seq.norm_rotate(q, k, None, None, None, f)
    assert [t._version for t in (q, k, v, g, S, f)] == before
    with pytest.raises(seq.PerError):       # refused: nothing is written
        seq.linear_attention(q, k, v, g, S, out=q)
    assert q._version == before[0]
    with torch.inference_mode():
        T = S.clone()
    seq.linear_attention_step(*(t[:, :1] for t in (q, k, v)), g, T)     # (these have no versions)


def test_inputs_that_ask_for_gradients_get_them():
    """The plain calls are nodes of the graph too where an input asks for a gradient: no result is detached without an error."""
    B, L, H, G, d = 2, 21, 4, 2, 32
    q, k, v, g, S, lengths = attention_inputs(B, L, H, G, d, d, F32, ragged=True)
    f, _ = seq.rotary_frequencies(d)
    w = 1 + 0.1 * normal(9, d)
    at = torch.arange(L, dtype=torch.int32, device="cuda").expand(B, L) + 7
    for i in range(4):      # one at a time
        ts = [q, k, v, S]
        ts[i], = leaves(ts[i])
        out, last = seq.linear_attention(*ts[:3], g, ts[3], lengths, scale=0.3)
        dout, dS = normal(11, *out.shape), normal(12, *S.shape)
        torch.autograd.backward((out, last), (dout, dS))
        assert torch.equal(ts[i].grad, seq.linear_attention_backward(dout, q, k, v, g, S, dS, lengths, scale=0.3)[i])
    a, = leaves(q)
    out, none = seq.linear_attention(a, k, v, g, S, lengths, want_state=False)
    assert none is None and torch.equal(out.detach(), seq.linear_attention(q, k, v, g, S, lengths)[0])
    out.sum().backward()
    assert torch.equal(a.grad, seq.linear_attention_backward(torch.ones_like(q), q, k, v, g, S, None, lengths)[0])
    for i in range(4):
        ts = [q, k, w, w]
        ts[i], = leaves(ts[i])
        x, y = seq.norm_rotate(*ts, at, f, eps=1e-3, layout="interleaved", magnitude=1.2)
        torch.autograd.backward((x, y), (normal(13, *q.shape), normal(14, *k.shape)))
        want = seq.norm_rotate_backward(normal(13, *q.shape), normal(14, *k.shape), q, k, w, w, at, f, eps=1e-3, layout="interleaved", magnitude=1.2)
        assert torch.equal(ts[i].grad, want[i])
    # (values below 6, two turns that round by 4 e each way: within 1e-5)
    for inverse in (False, True):
        for layout in ("half", "interleaved"):
            x, = leaves(q)
            y = seq.rotate(x, at, f, layout, 1.2, inverse)
            assert torch.equal(y.detach(), seq.rotate(q, at, f, layout, 1.2, inverse))
            first, = torch.autograd.grad((y * y).sum() / 2, x, create_graph=True)     # the magnitude twice, turned and back
            assert float((first.detach() - 1.2 ** 2 * q).abs().max()) < 1e-5
            again, = torch.autograd.grad(first, x, normal(13, *q.shape))
            assert float((again - 1.2 ** 2 * normal(13, *q.shape)).abs().max()) < 1e-5
    x, = leaves(q)
    seq.rotate(x, at, f).sum().backward()       # (a gradient whose last dimension is not contiguous)
    assert torch.equal(x.grad, seq.rotate(torch.ones_like(q), at, f, inverse=True))


def test_no_gradient_is_formed_where_none_is_asked_for():
    q, k, v, g, S, _ = attention_inputs(2, 9, 2, 2, 16, 16, F32)
    f, _ = seq.rotary_frequencies(16)
    with torch.no_grad():
        a, b, c = leaves(q, k, v)
        for t in (*seq.linear_attention(a, b, c, g, S), *seq.norm_rotate(a, b, None, None, None, f), seq.rotate(a, None, f),
                  seq.linear_attention_step(*(t[:, :1] for t in (a, b, c)), g, S)):
            assert not t.requires_grad
        seq.rotate(a, None, f, out=a)
    for t in (*seq.linear_attention(q, k, v, g, S), seq.rotate(q, None, f)):
        assert not t.requires_grad


def test_results_that_are_given_take_no_part_in_a_gradient():
    """Written over, they cannot be nodes of the graph: refused, as torch refuses it."""
    q, k, v, g, S, _ = attention_inputs(2, 1, 2, 2, 16, 16, F32)
    f, _ = seq.rotary_frequencies(16)
    a, T = leaves(q, S)
    room, room_state, b = torch.empty_like(q), torch.empty_like(S), a * 1.0
    before = b.detach().clone()
    refused = {
        "out": lambda: seq.linear_attention(a, k, v, g, S, out=room),
        "out_state": lambda: seq.linear_attention(a, k, v, g, S, out_state=room_state),
        "out itself": lambda: seq.linear_attention(q, k, v, g, S, out=a),
        "a step": lambda: seq.linear_attention_step(a, k, v, g, S),
        "a step's state": lambda: seq.linear_attention_step(q, k, v, g, T),
        "a step's out": lambda: seq.linear_attention_step(q, k, v, g, S, out=a),
        "rotate": lambda: seq.rotate(b, None, f, out=b),
        "q_out": lambda: seq.norm_rotate(a, k, None, None, None, f, q_out=room),
        "k_out": lambda: seq.norm_rotate(k, q, None, None, None, f, k_out=a),
    }
    for name, call in refused.items():
        with pytest.raises(RuntimeError, match="gradient"):
            call()
            print("not refused:", name)
    assert torch.equal(b, before)
