"""Sequences in bfloat16 by the 2-norm of their error: where states carry far, the bounds of single elements (sums of absolute values) are as
large as the outputs, and would pass much.

An output is the sum of two parts, from the state its chunk starts from and from the chunk's own tokens.  In each part one factor may be
rounded to bfloat16, and the output is: errors that are spread evenly within half a unit in the last place, at most 2^-8 / sqrt(3) of the
value as a root mean square.  Those of many products add up as their squares do, so that over many outputs the error is within
sqrt(2 / 3) 2^-8 = 3.2e-3 of them; allowed are 4e-3.  States are fp32 sums: (64 + L / 16) 2^-24 of the sum of absolute values bounds
each element (test_sequence.py), and the norm is held to 1e-5."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import sequence_oracle as oracle  # noqa: E402
from test_sequence import BF16, attention_inputs, normal  # noqa: E402
from paper_2311_09445_amd import sequence as seq  # noqa: E402

OFF, OFF_STATE, CHUNK = 4e-3, 1e-5, 32


def off(got, want):
    return float((got.detach().cpu().double() - want).norm() / want.norm())


def check_rows(got, want, what):
    """[B, L, H, d]: each head by itself, over all tokens, over those at the chunks' starts (which the states reach most), those at
    their ends, and the last 64."""
    for h in range(got.shape[2]):
        for name, at in (("all", slice(None)), ("starts", slice(0, None, CHUNK)), ("ends", slice(CHUNK - 1, None, CHUNK)), ("last", slice(-64, None))):
            x, y = got[:, at, h], want[:, at, h]
            if y.count_nonzero() >= 256:
                assert off(x, y) <= OFF, (what, h, name, off(x, y))


@pytest.mark.parametrize("B,L,H,G,dk,dv,fast,slow", [
    (1, 5003, 2, 1, 64, 48, 0.5, 2 ** -10),         # segments; a decay that carries a thousand tokens
    (1, 2000, 2, 2, 128, 128, 0.02, 2 ** -9),
    (2, 300, 4, 4, 64, 64, 0.5, 2 ** -8),
    (3, 1001, 2, 2, 64, 64, 0.1, 2 ** -9),
    (8, 160, 4, 4, 128, 128, 0.1, 2 ** -8),
    (1, 1500, 2, 1, 127, 113, 0.1, 2 ** -9),        # nothing in pieces of 16 bytes
    (1, 700, 2, 2, 5, 7, 0.1, 2 ** -8),
    (40, 96, 8, 2, 64, 64, 0.1, 2 ** -8),           # heads that share a key summed within a workgroup
    (40, 96, 8, 4, 32, 48, 0.1, 2 ** -8),
    (2, 2000, 4, 1, 32, 32, 0.1, 2 ** -9),          # and behind it
])
def test_norms(B, L, H, G, dk, dv, fast, slow):
    q, k, v, _, S, _ = attention_inputs(B, L, H, G, dk, dv, BF16)
    g = -torch.logspace(0, 1, H, base=slow / fast).float().cuda() * fast
    dout, dS = normal(11, B, L, H, dv, dtype=BF16), normal(12, B, H, dk, dv)
    few = min(B, 3)
    first = [t[:few] for t in (q, k, v)]
    want, want_state = oracle.attention(*first, g, S[:few], None, 0.3)
    out, last = seq.linear_attention(q, k, v, g, S, scale=0.3)
    check_rows(out[:few], want, "out")
    assert off(last[:few], want_state) <= OFF_STATE
    alone, _ = seq.linear_attention(q, k, v, g, S, scale=0.3, want_state=False)
    check_rows(alone[:few], want, "out without a state")
    got = seq.linear_attention_backward(dout, q, k, v, g, S, dS, scale=0.3)
    want = oracle.attention_backward(dout[:few], *first, g, S[:few], dS[:few], None, 0.3)
    for name, x, y in zip(("dq", "dk", "dv"), got, want):
        check_rows(x[:few], y, name)
    assert off(got[3][:few], want[3]) <= OFF_STATE
