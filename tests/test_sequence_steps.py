"""Single tokens of linear attention over thousands of steps, as an actor takes them.

Each step rounds what is left of a state and its sum with what is added, by at most e = 2^-24 each and now up, now down: after n steps
the error is within 8 sqrt(2 n) e A, A the state with every factor replaced by its absolute value (the rounding of a sum is at most e,
a root mean square of 0.6 e: 8 are thirteen of those)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from sequence_oracle import U_F32  # noqa: E402
from test_sequence import BF16, F32, normal, within  # noqa: E402
from paper_2311_09445_amd import sequence as seq  # noqa: E402


@pytest.mark.parametrize("d", [16, 5], ids=["vectors", "elements"])
@pytest.mark.parametrize("added", [False, True])
def test_slow_decays_do_not_drift(added, d):
    n, B, H, every = 20000, 2, 4, 100
    g = torch.tensor([-1e-5, -1e-4, -2.0 ** -8, -1.0], device="cuda")
    S = normal(1, B, H, d, d)
    q = normal(2, B, 1, H, d)
    k, v = (normal(i, B, every, H, d) if added else torch.zeros(B, every, H, d, device="cuda") for i in (3, 4))
    want, A = S.cpu().double(), S.cpu().double().abs()
    decay = torch.exp(g.cpu().double())[:, None, None]
    terms = torch.einsum("bthi,bthj->tbhij", k.cpu().double(), v.cpu().double())
    for t in range(n):
        want = want * decay + terms[t % every]
        A = A * decay + terms[t % every].abs()
        seq.linear_attention_step(q, k[:, t % every:t % every + 1], v[:, t % every:t % every + 1], g, S)
    within(S, want, 8 * (2 * n) ** 0.5 * U_F32 * A, "state")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_steps_reach_the_state_that_the_sequence_does(dtype):
    """What actors carry is what a learner computes from the same tokens: 2000 steps, both within their bounds of each other."""
    n, B, H, d = 2000, 2, 3, 32
    g = torch.tensor([-2.0 ** -12, -2.0 ** -7, -0.5], device="cuda")
    q, k, v = (normal(i, B, n, H, d, dtype=dtype) for i in (2, 3, 4))
    S = normal(1, B, H, d, d)
    T, A = S.clone(), S.cpu().double().abs()
    decay = torch.exp(g.cpu().double())[:, None, None]
    for t in range(n):
        seq.linear_attention_step(*(x[:, t:t + 1] for x in (q, k, v)), g, T)
        A = A * decay + k[:, t].cpu().double().abs()[..., None] * v[:, t].cpu().double().abs()[..., None, :]
    _, last = seq.linear_attention(q, k, v, g, S)
    within(T, last.cpu().double(), (8 * (2 * n) ** 0.5 + 64 + n / 16) * U_F32 * A, "state")


def test_refusals_name_the_argument():
    q, S = normal(2, 3, 1, 2, 16), normal(1, 3, 2, 16, 16)
    g = torch.tensor([-0.1, -0.2], device="cuda")
    for active in (torch.ones(2, dtype=torch.int32, device="cuda"), torch.ones(3, device="cuda"), torch.ones(3, dtype=torch.int32)):
        with pytest.raises(ValueError, match="active"):
            seq.linear_attention_step(q, q, q, g, S, active)
        with pytest.raises(ValueError, match="lengths"):
            seq.linear_attention(q, q, q, g, S, active)
    with pytest.raises(TypeError, match="active"):
        seq.linear_attention_step(q, q, q, g, S, [1, 0, 1])
