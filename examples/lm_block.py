"""A small transformer trained through the package: embedding, blocks of layer norm, self-attention with rotary positions and an MLP, all linear layers with MVUE 2:4 pruned
weight gradients, AdamW with 8-bit states.  Sequences of a batch differ in length.

The model predicts the next token of a fixed random rule of the last two.  python examples/lm_block.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2203_10991_amd.autograd import NMConfig, NMEmbedding, NMLayerNorm, NMLinear, NMLinearReLU, NMSelfAttention  # noqa: E402
from paper_2203_10991_amd.optim import NMAdamW  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, width: int, heads: int, kv_heads: int, cfg: NMConfig, **kw):
        super().__init__()
        self.norm1, self.attn = NMLayerNorm(width, **kw), NMSelfAttention(width, heads, kv_heads, cfg=cfg, **kw)
        self.norm2, self.up, self.down = NMLayerNorm(width, **kw), NMLinearReLU(width, 4 * width, cfg=cfg, **kw), NMLinear(4 * width, width, cfg=cfg, **kw)

    def forward(self, x, lens=None):
        x = x + self.attn(self.norm1(x), lens=lens)
        return x + self.down(self.up(self.norm2(x)))


class Model(torch.nn.Module):
    def __init__(self, vocab: int, width: int, layers: int, heads: int, kv_heads: int, cfg: NMConfig, **kw):
        super().__init__()
        self.embed = NMEmbedding(vocab, width, scale=width ** 0.5, **kw)
        torch.nn.init.normal_(self.embed.weight, std=width ** -0.5)
        self.blocks = torch.nn.ModuleList(Block(width, heads, kv_heads, cfg, **kw) for _ in range(layers))
        self.norm, self.head = NMLayerNorm(width, **kw), NMLinear(width, vocab, cfg=cfg, **kw)

    def forward(self, ids, lens=None):
        x = self.embed(ids)
        for block in self.blocks:
            x = block(x, lens)
        return self.head(self.norm(x))


def loss_of(model, ids, target, lens):
    there = torch.arange(ids.shape[1], device=ids.device) < lens[:, None]
    return F.cross_entropy(model(ids, lens).float().flatten(0, 1), torch.where(there, target, -100).flatten(), ignore_index=-100)


def train(steps: int = 60, vocab: int = 256, width: int = 256, layers: int = 2, heads: int = 8, kv_heads: int = 2, batch: int = 32, length: int = 64, dtype=torch.bfloat16,
          device: str = "cuda:0"):
    """Losses of `steps` training steps."""
    torch.manual_seed(0)
    cfg = NMConfig(seed=1)
    model = Model(vocab, width, layers, heads, kv_heads, cfg, device=device, dtype=dtype)
    opt = NMAdamW(model.parameters(), lr=2e-3, weight_decay=0.01, states="q8", master=True, seed=2)
    rule = torch.randint(vocab, (16, 16), device=device)                  # the next token, by the last two modulo 16
    losses = []
    for _ in range(steps):
        ids = torch.randint(vocab, (batch, length), device=device)
        before = torch.cat((torch.zeros_like(ids[:, :1]), ids[:, :-1]), 1)
        lens = torch.randint(length // 2, length + 1, (batch,), dtype=torch.int32, device=device)
        opt.zero_grad()
        loss = loss_of(model, ids, rule[ids % 16, before % 16], lens)
        loss.backward()
        norm = torch.stack([p.grad.float().norm() for p in model.parameters()]).norm()
        opt.step(grad_scale=(1.0 / norm.clamp(min=1.0)).reshape(1))       # the clip's coefficient stays on the device
        cfg.advance()
        losses.append(loss.detach())
    return [float(x) for x in losses]


if __name__ == "__main__":
    out = train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
    for k in range(0, len(out), max(1, len(out) // 10)):
        print(f"step {k:4d}  loss {out[k]:.4f}")
    print(f"last       loss {out[-1]:.4f}")
