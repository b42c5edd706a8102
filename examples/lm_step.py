"""A small language model trained through the package: embedding lookup and its gradient by sorted tokens, linear layers whose dense products are in 8-bit
integers and whose weight gradients are MVUE 2:4 pruned, AdamW with 8-bit states and binary32 master weights.

The model sees a token and its predecessor and predicts the next one; the data is a fixed random rule of both.  python examples/lm_step.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2203_10991_amd.autograd import NMConfig, NMEmbedding, NMLinear, NMLinearReLU  # noqa: E402
from paper_2203_10991_amd.optim import NMAdamW  # noqa: E402


class TokenModel(torch.nn.Module):
    def __init__(self, vocab: int, width: int, cfg: NMConfig, device, dtype=torch.bfloat16):
        super().__init__()
        kw = dict(device=device, dtype=dtype)
        self.embed = NMEmbedding(vocab, width, scale=width ** 0.5, **kw)
        torch.nn.init.normal_(self.embed.weight, std=width ** -0.5)
        self.up, self.down = NMLinearReLU(2 * width, 4 * width, cfg=cfg, **kw), NMLinear(4 * width, width, cfg=cfg, **kw)
        self.head = NMLinear(width, vocab, cfg=cfg, **kw)

    def forward(self, ids):
        x = self.embed(ids)                                              # [batch, length, width]
        x = torch.cat((x[:, 1:], x[:, :-1]), -1)
        return self.head(F.rms_norm(self.down(self.up(x)), (x.shape[-1] // 2,)))


def train(steps: int = 60, vocab: int = 256, width: int = 256, batch: int = 32, length: int = 65, dense: str = "i8", states: str = "q8", device: str = "cuda:0"):
    """Losses of `steps` training steps."""
    torch.manual_seed(0)
    cfg = NMConfig(seed=1, dense=dense)
    model = TokenModel(vocab, width, cfg, device)
    opt = NMAdamW(model.parameters(), lr=2e-3, weight_decay=0.01, states=states, master=True, seed=2)
    rule = torch.randint(vocab, (16, 16), device=device)                  # the next token, by the last two modulo 16
    losses = []
    for _ in range(steps):
        ids = torch.randint(vocab, (batch, length), device=device)
        target = rule[ids[:, 1:] % 16, ids[:, :-1] % 16]
        opt.zero_grad()
        loss = F.cross_entropy(model(ids).float().flatten(0, 1), target.flatten())
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
