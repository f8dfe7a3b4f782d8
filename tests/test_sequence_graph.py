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
