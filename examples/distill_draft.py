"""Drafting, verifying and learning from the verdicts, with random weights.

A target head and a draft head read the same hidden states, the draft's
through a narrow projection of its own.  Each step:

  1. the draft's tokens are drawn from its logits (``sample``);
  2. the target's rows verify them (``verify``), which gives the accepted counts;
  3. the target's largest logits at the drafted positions are kept (``top_logits``);
  4. the draft head is trained on them (``distill``), so that more of the next
     step's drafts are accepted.

    python examples/distill_draft.py --steps 60
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_01083_amd as dsde  # noqa: E402


def run(steps=60, B=64, sl=4, V=8000, hidden=64, narrow=48, K=32, T=1.0, lr=0.02, seed=0, report=print):
    """Returns (accepted drafts per sequence, mean loss) of every step."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev)

    w_target = 0.4 * randn(hidden, V)
    down, up = (0.1 * randn(hidden, narrow)).requires_grad_(), (0.1 * randn(narrow, V)).requires_grad_()
    optimizer = torch.optim.Adam([down, up], lr=lr)
    N, k_max = B * sl, sl
    lengths = torch.full((B,), sl, dtype=torch.int32, device=dev)
    cu = torch.arange(0, N + 1, sl, dtype=torch.int32, device=dev)
    temperature = torch.full((B,), T, device=dev)
    # target row of drafted position (b, j); row b * (sl + 1) + sl is the bonus row
    rows = (torch.arange(N, device=dev) + torch.arange(N, device=dev) // sl)
    verify_ws = dsde.new_workspace(B, N, V, k_max)
    rows_ws = dsde.new_sample_workspace(N, V)
    history = []
    for step in range(steps):
        states = randn(N + B, hidden)
        target = states @ w_target
        logits = states[rows] @ down @ up
        drawn = dsde.sample(logits.detach(), temperature.repeat_interleave(sl), torch.rand(N, generator=g, device=dev),
                            workspace=rows_ws)
        verdict = dsde.verify(target, logits.detach(), lengths, cu, drawn["tokens"], temperature,
                              torch.rand(N, generator=g, device=dev), torch.rand(B, generator=g, device=dev), k_max,
                              workspace=verify_ws)
        teacher = dsde.top_logits(target[rows], K, temperature=T, workspace=rows_ws)
        loss = dsde.distill(logits, teacher["ids"], teacher["values"], teacher["lse"], T).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        history.append((verdict["accepted"].float().mean(), loss.detach()))
        if report and (step % 10 == 0 or step == steps - 1):
            report(f"step {step:4d}  accepted {float(history[-1][0]):.2f} of {sl}  loss {float(history[-1][1]):.4f}")
    return [(float(a), float(b)) for a, b in history]


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    run(steps=a.steps, seed=a.seed)
