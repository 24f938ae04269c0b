"""A small mixture of experts in microscaled 4-bit floating point: trained for a few steps, then served.

    python examples/mx4_experts.py [--steps 30] [--tokens 2048] [--hidden 512] [--ffn 1024] [--experts 8]

The experts' two projections are `mx4.experts` layers: rows sorted by expert, any number for each, gradients of rows and weights; what they keep
for the backward pass is 4.25 bits a value.  Around them `SavedActivationCompression` keeps what the other operators save (here the gate's
activations) in 4-bit codes with outliers.  Serving keeps the weights as `Mx4Matrix` and takes a few tokens at a time.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2508_00806_amd import OUTLIER_TOPK, Method, mx4  # noqa: E402
from paper_2508_00806_amd.hooks import SavedActivationCompression  # noqa: E402


class Experts(torch.nn.Module):
    """x + sum over the top two experts of share * down(silu(up(x)))"""

    def __init__(self, hidden, ffn, experts, seed=0):
        super().__init__()
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *shape, s: torch.nn.Parameter(torch.randn(*shape, generator=g, device="cuda") * s)
        self.route = draw(experts, hidden, s=hidden ** -0.5)
        self.up = draw(experts, ffn, hidden, s=hidden ** -0.5)
        self.down = draw(experts, hidden, ffn, s=ffn ** -0.5)

    def sorted_by_expert(self, x):
        """(row of x, its share, offsets of the experts) for the rows that the experts take, expert after expert; nothing waits for the GPU."""
        share, chosen = torch.softmax(x.float() @ self.route.t(), -1).topk(2)
        order = chosen.flatten().argsort(stable=True)
        counts = torch.zeros(self.route.shape[0] + 1, dtype=torch.int32, device=x.device)
        counts[1:] = (chosen.flatten()[:, None] == torch.arange(self.route.shape[0], device=x.device)).sum(0)
        return order // 2, share.flatten()[order], counts.cumsum(0, dtype=torch.int32)

    def forward(self, x, up=None, down=None):
        row, share, offsets = self.sorted_by_expert(x)
        h = mx4.experts(x[row], offsets, self.up if up is None else up)
        h = mx4.experts(F.silu(h), offsets, self.down if down is None else down)
        return x + torch.zeros_like(x).index_add(0, row, (h * share[:, None]).to(x.dtype))


def policy(t):
    """INT4 with the four largest of 1024 values kept, for whatever autograd saves of the gates' activations."""
    if t.numel() % 1024:
        return None
    return Method(bits=4, quant_group=128, outlier_mode=OUTLIER_TOPK, stat_group=1024, topk=4, max_outliers=4 * t.numel() // 1024 + 64)


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("steps", 30), ("tokens", 2048), ("hidden", 512), ("ffn", 1024), ("experts", 8)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    torch.manual_seed(0)
    model, teacher = Experts(a.hidden, a.ffn, a.experts, 1), Experts(a.hidden, a.ffn, a.experts, 2)
    teacher.route.data.copy_(model.route.data)
    optimiser = torch.optim.Adam([model.up, model.down], lr=3e-3)
    losses = []
    for step in range(a.steps):
        x = torch.randn(a.tokens, a.hidden, device="cuda", dtype=torch.bfloat16)
        with torch.no_grad():
            want = teacher(x)
        saved = SavedActivationCompression(policy, timing=False)
        with saved:
            loss = (model(x) - want).float().square().mean()
            loss.backward()
        optimiser.step()
        optimiser.zero_grad(set_to_none=True)
        losses.append(loss.detach())
    losses = [float(v) for v in losses]
    print(f"training: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps; {len(saved.records)} activations a step by the hooks")

    up, down = mx4.compress(model.up), mx4.compress(model.down)
    plain = 4 * (model.up.numel() + model.down.numel())
    with torch.no_grad():
        x = torch.randn(64, a.hidden, device="cuda", dtype=torch.bfloat16)
        whole = model(x)
        served = model(x, up, down)
        one = torch.cat([model(x[i:i + 1], up, down) for i in range(4)])
    assert torch.equal(served, whole)  # the layer compresses its weights to the same codes
    err = float((one.float() - whole[:4].float()).abs().max())
    print(f"serving: {plain / 2 ** 20:.1f} MiB of weights in {(up.nbytes + down.nbytes) / 2 ** 20:.1f} MiB; token by token differs by {err:.1e} at most")
    return losses, err


if __name__ == "__main__":
    main()
