"""The sequence operators on values that are not finite: they reach all that depends on them, whichever way a sequence is computed."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import sequence_oracle as oracle  # noqa: E402
from test_sequence import BF16, F32, attention_inputs, normal  # noqa: E402
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
