"""The feed-forward half of a transformer block in int8, served and trained with the package's operators.

    python examples/int8_ffn_block.py [--tokens 1576] [--width 768] [--hidden 2048] [--steps 20]

Serving (one pass): the norm before the block leaves int8 codes, the gated block reads them, its product back to the
residual's width (a 2:4 sparse weight) reads codes of the hidden activations, and the next block's norm takes the sum.
Training (one step): the same block with dense weights in float32 masters, quantised every step; the gradients pass
straight through the codes.  The example fits the block to a fixed random target and prints the loss.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_12505_amd import nmblock as nb  # noqa: E402


def prune(w, N, M):
    """int8 codes and scales of w with the N largest of each M consecutive weights kept."""
    groups = w.view(w.shape[0], -1, M)
    drop = groups.abs().topk(M - N, dim=2, largest=False).indices
    q, scale = nb.quantize_rows(groups.scatter(2, drop, 0.0).view_as(w))
    return q, scale


class ServedFfn:
    """norm -> gated block -> 2:4 product -> gate, residual and the next norm."""

    def __init__(self, width, hidden, device="cuda", dtype=torch.float16):
        f32 = dict(device=device, dtype=torch.float32)
        self.norm = nb.Norm("layer", torch.ones(width, **f32), torch.zeros(width, **f32))
        self.next_norm = nb.Norm("layer", torch.ones(width, **f32), torch.zeros(width, **f32))
        wg, wu = (torch.randn(hidden, width, **f32) * width ** -0.5 for _ in range(2))
        self.gated = nb.GatedWeight.from_float(wg, wu, act="silu")
        q, scale = prune(torch.randn(width, hidden, **f32) * hidden ** -0.5, 2, 4)
        self.down = nb.ScaledWeight.from_int8(q[:, :hidden], scale, N=2, M=4)
        self.gate = torch.full((width,), 0.5, **f32)
        self.dtype = dtype

    def __call__(self, attention, residual):
        residual, codes, scales = nb.norm_residual_i8(attention, residual, pre=self.norm)
        hidden = nb.gated_ffn_i8(codes, scales, self.gated, out_dtype=self.dtype)
        return nb.norm_residual(nb.linear_i8(hidden, self.down), residual, pre=self.next_norm, gate=self.gate)


class TrainedGate:
    """A norm and a gated block with float32 masters, trained through their int8 codes."""

    def __init__(self, width, hidden, device="cuda"):
        f32 = dict(device=device, dtype=torch.float32)
        self.wg, self.wu = (torch.randn(hidden, width, **f32) * width ** -0.5 for _ in range(2))
        self.norm = nb.Norm("rms", torch.ones(width, **f32))

    def step(self, x, target, rate):
        weight = nb.GatedWeight.from_float(self.wg, self.wu)          # this step's codes
        residual, codes, scales = nb.norm_residual_i8(None, x, pre=self.norm)
        h = nb.gated_ffn_i8(codes, scales, weight, out_dtype=x.dtype)
        off = h.float() - target
        loss = off.square().mean()
        dh = (off * (2.0 * 1024 / h.shape[0])).to(x.dtype)            # of 1024 * (sum of squares) / tokens
        grads = nb.gated_ffn_backward(codes, scales, weight, dh)
        through = nb.norm_residual_backward(grads.dx, None, None, residual, pre=self.norm)
        self.wg.sub_(grads.dw_gate.float(), alpha=rate / 1024)
        self.wu.sub_(grads.dw_up.float(), alpha=rate / 1024)
        # one value serves every hidden unit: its gradient is the sum of all of theirs
        self.norm.weight.sub_(through.dpre_weight, alpha=rate / (1024 * target.shape[1]))
        return loss


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=1576)
    ap.add_argument("--width", type=int, default=768)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    torch.manual_seed(0)
    served = ServedFfn(args.width, args.hidden)
    for tokens in (1, args.tokens):
        y, r = (torch.randn(tokens, args.width, device="cuda", dtype=torch.float16) for _ in range(2))
        residual, z = served(y, r)
        assert torch.isfinite(residual).all() and torch.isfinite(z).all()
        print(f"served {tokens} tokens: residual {tuple(residual.shape)}, next norm's rows within "
              f"{z.float().abs().max().item():.2f}")
    trained = TrainedGate(args.width, args.hidden)
    x = torch.randn(args.tokens, args.width, device="cuda", dtype=torch.bfloat16)
    target = 0.5 * torch.randn(args.tokens, args.hidden, device="cuda")
    losses = [trained.step(x, target, rate=0.1).item() for _ in range(args.steps)]
    print("loss " + " ".join(f"{v:.4f}" for v in losses))
    assert losses[-1] < losses[0]
    return losses


if __name__ == "__main__":
    main()
