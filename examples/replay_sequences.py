"""Actors and a learner of sequences around one prioritized replay buffer.

Actors read a stream of observations token by token (``linear_attention_step``: a state of fixed size per actor) and record
stretches of it: observations, targets, the number of valid steps, the position and the state each stretch started from.  Stretches
are rows of the buffer.  The learner samples rows, runs its policy over the whole stretches from the states stored with them
(``norm_rotate`` and ``linear_attention`` with their gradients), weighs the errors with the importance weights, and hands the
errors back as priorities.

The stream is synthetic: the target is a decayed sum of a hidden projection of the observations, which a policy without memory
cannot tell.

    python examples/replay_sequences.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2311_09445_amd import sequence as seq  # noqa: E402
from paper_2311_09445_amd.per import PrioritizedReplay  # noqa: E402

ACTORS, STRETCH, BATCH = 64, 40, 128
WIDTH, HEADS, KV_HEADS, HEAD = 16, 4, 2, 32
MEMORY = 0.9          # what the target keeps from step to step


class Policy(torch.nn.Module):
    """Observations to predictions through one layer of linear attention."""

    def __init__(self):
        super().__init__()
        wide, shared = HEADS * HEAD, KV_HEADS * HEAD
        self.q, self.k, self.v = (torch.nn.Linear(WIDTH, n) for n in (wide, shared, shared))
        self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(HEAD)) for _ in range(2))
        self.out = torch.nn.Linear(wide, 1)
        self.register_buffer("log_decay", -torch.tensor([0.05, 0.1, 0.2, 0.4]))
        self.register_buffer("freqs", seq.rotary_frequencies(HEAD // 2, base=1000.0, device="cpu")[0])   # half of each head turns

    def rows(self, x):
        return (f(x).unflatten(-1, (-1, HEAD)).bfloat16() for f in (self.q, self.k, self.v))

    def forward(self, x, positions, state, lengths):
        q, k, v = self.rows(x)
        q, k = seq.norm_rotate_autograd(q, k, self.q_weight, self.k_weight, positions, self.freqs)
        o, _ = seq.linear_attention_autograd(q, k, v, self.log_decay, state, lengths)
        return self.out(o.float().flatten(-2))[..., 0]

    @torch.no_grad()
    def step(self, x, positions, state):
        """One token of every actor; ``state`` is advanced in place."""
        q, k, v = self.rows(x[:, None])
        q, k = seq.norm_rotate(q, k, self.q_weight, self.k_weight, positions[:, None], self.freqs)
        o = seq.linear_attention_step(q, k, v, self.log_decay, state)
        return self.out(o.float().flatten(-2))[:, 0, 0]


class Stream:
    """What the actors see, and the targets of it."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden = torch.randn(WIDTH, generator=self.g, device="cuda") / WIDTH ** 0.5
        self.sum = torch.zeros(ACTORS, device="cuda")

    def next(self):
        x = torch.randn(ACTORS, WIDTH, generator=self.g, device="cuda")
        self.sum = MEMORY * self.sum + x @ self.hidden
        return x, self.sum


def as_bytes(t):
    """[n, ...] -> the [1, n, bytes] that a field of the buffer takes."""
    return t.contiguous().reshape(t.shape[0], -1).view(torch.uint8)[None]


def main(iterations=150, seed=0, report=print):
    torch.manual_seed(seed)
    policy, stream = Policy().cuda(), Stream(seed)
    optimiser = torch.optim.Adam(policy.parameters(), 1e-2)
    shapes = [((STRETCH, WIDTH), torch.float32), ((STRETCH,), torch.float32), ((HEADS, HEAD, HEAD), torch.float32),
              ((1,), torch.int32), ((1,), torch.int32)]   # observations, targets, state at the start, valid steps, position of the first
    widths = [4 * torch.Size(s).numel() for s, _ in shapes]
    buffer = PrioritizedReplay(16, 8192, 1, widths)
    buffer.set_rng(seed)
    rows = [torch.empty(1, BATCH, w, dtype=torch.uint8, device="cuda") for w in widths]
    state = torch.zeros(ACTORS, HEADS, HEAD, HEAD, device="cuda")
    position = torch.zeros(ACTORS, dtype=torch.int32, device="cuda")
    losses = []
    for i in range(iterations):
        # actors: a stretch each, some cut short
        start, first, seen, targets, errors = state.clone(), position.clone(), [], [], []
        for _ in range(STRETCH):
            x, y = stream.next()
            errors.append((policy.step(x, position, state) - y).abs())
            seen.append(x)
            targets.append(y)
            position += 1
        lengths = torch.randint(STRETCH // 2, STRETCH + 1, (ACTORS,), generator=stream.g, device="cuda", dtype=torch.int32)
        fields = (torch.stack(seen, 1), torch.stack(targets, 1), start, lengths[:, None], first[:, None])
        buffer.insert(ACTORS, [as_bytes(t) for t in fields])
        # learner: a batch of stretches by priority
        idx, weights, _ = buffer.sample(None, 0.4 + 0.6 * i / iterations, rows_out=rows, B=BATCH)
        x, y, s, n, p = (r[0].view(dtype).reshape(BATCH, *shape) for r, (shape, dtype) in zip(rows, shapes))
        steps = torch.arange(STRETCH, dtype=torch.int32, device="cuda")
        here = steps < n
        error = (policy(x, p + steps, s, n[:, 0].contiguous()) - y) * here
        per_row = error.square().sum(1) / n[:, 0]
        optimiser.zero_grad()
        (weights[0] * per_row).mean().backward()
        optimiser.step()
        buffer.update_td(idx, per_row.detach().sqrt()[None].contiguous())
        losses.append(torch.stack(errors).square().mean())      # of the actors, on what they had not seen before
        if report and i % 25 == 24:
            report(f"iteration {i + 1}: mean square error of the actors {float(losses[-1]):.4f}")
    assert buffer.status() == 0
    return [float(x) for x in losses]


if __name__ == "__main__":
    main()
