"""Training steps of a small language model on the library's operators, start to end:

  embedding lookup -> linear layers in 8-bit floating point -> loss
  -> neural gradients pruned by their lognormal statistics -> input and weight gradients in 8-bit floating point
  -> table gradient by sorted tokens -> clipping by the global norm -> update

The task is synthetic: the next token is a fixed permutation of the current one, nine times in ten.

    python examples/lm_step.py [--steps 60] [--sparsity 0.5]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2006_08173_b200.layers import Embedding, Fp8Linear, GradClipper  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, vocab: int, dim: int, hidden: int, sparsity: float):
        super().__init__()
        self.embed = Embedding(vocab, dim, scale=dim ** 0.5, device="cuda")
        self.up = Fp8Linear(dim, hidden, sparsity, device="cuda", seed=1 << 32)
        self.down = Fp8Linear(hidden, dim, sparsity, device="cuda", seed=2 << 32)
        self.head = Fp8Linear(dim, vocab, device="cuda")

    def forward(self, ids: torch.Tensor) -> torch.Tensor:
        x = self.embed(ids)
        x = x + self.down(torch.nn.functional.gelu(self.up(x)))
        return self.head(x)


def train(steps: int = 60, sparsity: float = 0.5, vocab: int = 1000, dim: int = 256, hidden: int = 640, tokens: int = 2048,
          max_norm: float = 1.0, seed: int = 0):
    """Losses and gradient norms of every step."""
    torch.manual_seed(seed)
    model = Model(vocab, dim, hidden, sparsity)
    opt = torch.optim.Adam(model.parameters(), lr=3e-3)
    follow = torch.randperm(vocab, device="cuda")
    clipper, losses, norms = None, [], []
    for _ in range(steps):
        ids = torch.randint(0, vocab, (tokens,), device="cuda")
        target = torch.where(torch.rand(tokens, device="cuda") < 0.9, follow[ids], torch.randint(0, vocab, (tokens,), device="cuda"))
        loss = torch.nn.functional.cross_entropy(model(ids).float(), target)
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
