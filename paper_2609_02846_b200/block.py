"""A pre-norm transformer block for training: the four linears of a layer (QKV, output projection, MLP up and down) in UE5M3-FP4
and between them the library's layer norm, attention and dropout-add.

    x = x + dropout(proj(attention(qkv(norm1(x)))))
    x = x + dropout(down(relu(up(norm2(x)))^2))

`python -m paper_2609_02846_b200.block` trains one block on synthetic data and prints the time of a step."""
from __future__ import annotations

import argparse
import time
from typing import Callable, Optional

import torch

from .autograd import DropoutAdd, LayerNorm, Ue5m3Linear, attention


class TransformerBlock(torch.nn.Module):
    """One pre-norm block over x [batch, tokens, hidden] (bfloat16), grouped-query attention.  `linear(in, out)` builds the four
    linears (Ue5m3Linear by default: tokens and widths must then be multiples of 128).  Call `advance()` once per optimizer step and, where
    gradients are accumulated, `next_micro_batch()` between the micro-batches of a step."""

    def __init__(self, hidden: int, heads: int, kv_heads: int, ffn: int, p: float = 0.1, window_left: int = -1,
                 linear: Optional[Callable] = None):
        super().__init__()
        if hidden % heads or heads % kv_heads:
            raise ValueError(f"hidden {hidden}, heads {heads} and kv_heads {kv_heads} do not divide")
        self.heads, self.kv_heads, self.head_dim, self.window_left = heads, kv_heads, hidden // heads, window_left
        linear = Ue5m3Linear if linear is None else linear
        self.norm1, self.norm2 = LayerNorm(hidden), LayerNorm(hidden)
        self.qkv = linear(hidden, (heads + 2 * kv_heads) * self.head_dim)
        self.proj = linear(hidden, hidden)
        self.up, self.down = linear(hidden, ffn), linear(ffn, hidden)
        self.drop1, self.drop2 = DropoutAdd(p), DropoutAdd(p)

    def advance(self) -> None:
        for m in self.children():
            if hasattr(m, "advance"):
                m.advance()

    def next_micro_batch(self) -> None:
        """New dropout masks; the linears stay at their step."""
        self.drop1.advance()
        self.drop2.advance()

    def forward(self, x: torch.Tensor, k_lens: Optional[torch.Tensor] = None) -> torch.Tensor:
        B, L, hidden = x.shape
        rows = x.reshape(B * L, hidden)
        qkv = self.qkv(self.norm1(rows)).view(B, L, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=2)          # views: no copy
        o = attention(q, k, v, causal=True, window_left=self.window_left, k_lens=k_lens)
        rows = self.drop1(self.proj(o.view(B * L, hidden)), rows)
        h = torch.relu(self.up(self.norm2(rows)))
        return self.drop2(self.down(h * h), rows).view(B, L, hidden)


def main() -> None:
    ap = argparse.ArgumentParser(description="Train one UE5M3-FP4 transformer block on synthetic data")
    ap.add_argument("--batch", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--ffn", type=int, default=16384)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args()
    torch.manual_seed(0)
    block = TransformerBlock(a.hidden, a.heads, a.kv_heads, a.ffn, a.dropout)
    opt = torch.optim.SGD(block.parameters(), lr=1e-2)
    x = torch.randn(a.batch, a.tokens, a.hidden, device="cuda", dtype=torch.bfloat16)
    target = torch.randn_like(x)
    for step in range(a.steps):
        torch.cuda.synchronize()
        t = time.perf_counter()
        loss = torch.nn.functional.mse_loss(block(x).float(), target.float())
        loss.backward()
        opt.step()
        opt.zero_grad(set_to_none=True)
        block.advance()
        torch.cuda.synchronize()
        print(f"step {step}: loss {loss.item():.4f}, {(time.perf_counter() - t) * 1e3:.2f} ms")


if __name__ == "__main__":
    main()
