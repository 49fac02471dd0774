"""Training steps of a small student that learns from a larger teacher's top logits, on the library's operators, start to end:

  embedding lookup -> rows sorted by expert -> two layers of experts -> output layer in 8-bit integers
  -> loss against the teacher's top logits and the labels -> neural gradients pruned by their lognormal statistics
  -> gradients of experts and output layer -> table gradient -> clipping by the global norm -> update

The teacher is a fixed table of logits per token; labels are its favourites.

    python examples/distill_step.py [--steps 60] [--sparsity 0.5]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2006_08173_b200.layers import DistillLoss, Embedding, ExpertLinear, GradClipper, Int8Linear, by_expert  # noqa: E402


class Student(torch.nn.Module):
    def __init__(self, vocab: int, dim: int, hidden: int, experts: int, chosen: int, sparsity: float):
        super().__init__()
        self.experts, self.chosen = experts, chosen
        self.embed = Embedding(vocab, dim, scale=dim ** 0.5, device="cuda")
        self.gate = torch.nn.Linear(dim, experts, bias=False, device="cuda")
        self.up = ExpertLinear(experts, dim, hidden, sparsity, device="cuda", seed=1 << 32)
        self.down = ExpertLinear(experts, hidden, dim, sparsity, device="cuda", seed=2 << 32)
        self.head = Int8Linear(dim, vocab, device="cuda")

    def forward(self, ids: torch.Tensor) -> torch.Tensor:
        x = self.embed(ids)
        share, expert = torch.softmax(self.gate(x.float()), dim=-1).topk(self.chosen)
        order, offsets = by_expert(expert.reshape(-1), self.experts)
        y = self.down(torch.nn.functional.gelu(self.up(x[order // self.chosen], offsets)), offsets)
        back = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=order.device))    # where each token's rows went
        y = (y[back].reshape(*expert.shape, -1) * share[..., None]).sum(dim=-2)
        return self.head((x + y).to(torch.bfloat16))


def train(steps: int = 60, sparsity: float = 0.5, vocab: int = 1000, dim: int = 256, hidden: int = 320, experts: int = 8, chosen: int = 2,
          tokens: int = 1024, top: int = 16, temperature: float = 2.0, alpha: float = 0.7, max_norm: float = 1.0, seed: int = 0):
    """Losses and gradient norms of every step."""
    torch.manual_seed(seed)
    model = Student(vocab, dim, hidden, experts, chosen, sparsity)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    logits, places = (3.0 * torch.randn(vocab, vocab, device="cuda")).topk(top)
    loss_of = DistillLoss(temperature, alpha)
    clipper, losses, norms = None, [], []
    for _ in range(steps):
        ids = torch.randint(0, vocab, (tokens,), device="cuda")
        loss = loss_of(model(ids), places[ids], logits[ids], places[ids, 0]).mean()
        opt.zero_grad(set_to_none=False)
        loss.backward()
        if clipper is None:
            clipper = GradClipper(list(model.parameters()), max_norm)
        norms.append(clipper.clip())
        opt.step()
        for layer in (model.up, model.down):
            layer.advance()
        losses.append(loss.detach())
    for layer in (model.up, model.down, model.head):
        layer.check()
    return torch.stack(losses).tolist(), torch.stack(norms).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--sparsity", type=float, default=0.5, help="zeros in the pruned neural gradients (0: no pruning)")
    args = ap.parse_args()
    loss, norm = train(args.steps, args.sparsity)
    for i in range(0, args.steps, max(1, args.steps // 10)):
        print(f"step {i:4d}  loss {loss[i]:.4f}  gradient norm {norm[i]:.4f}")
    print(f"last      loss {loss[-1]:.4f}  gradient norm {norm[-1]:.4f}")
