"""Fine-tuning and serving low-rank adapters on a frozen two-bit network.

``AdaptedStack`` is a chain of pre-norm residual blocks of one width

    x <- x + W~ h + scale_i b_i (a_i h),        h = layernorm(x)

whose square projections W~ are two-bit (quantized once, codes and alpha kept)
and whose adapters (a_i, b_i) are many requests' or tenants': every token says
in ``ids`` which one it takes, or none.  ``forward`` and ``backward`` are
library launches on the current stream; ``step`` updates all adapters and norm
weights with one AdamW launch, whose fp32 parameters write the bf16 copies that
the next forward reads, and keeps the adapters' moments in 8 bits.  With
``train=False`` forward keeps nothing and takes any number of tokens, so the
same call serves prompts and single tokens.

    python -m paper_1701_00485_gb300.finetune

learns random targets for a few adapters and prints the loss, then serves
single tokens with what was learnt.
"""
from __future__ import annotations

import argparse

import torch

from . import (AdamWPlan, packed_words, tbn_adamw_step, tbn_adapter_bwd, tbn_adapter_fwd,
               tbn_adapter_workspace_bytes, tbn_conv2d_bwd_data, tbn_layernorm_bwd,
               tbn_layernorm_fwd, tbn_linear_fwd, tbn_quantize_pack)
from . import inputs as _inputs


class AdaptedStack:
    """``depth`` blocks of width ``width`` with ``adapters`` adapters of rank
    ``rank`` each.  ids: int32 [tokens], values outside 0 .. adapters - 1 for
    tokens without one."""

    def __init__(self, width: int, depth: int, adapters: int, rank: int, seed: int = 0,
                 device="cuda"):
        g = _inputs.generator(seed)
        dev = torch.device(device)
        self.width, self.depth, self.n, self.r = width, depth, adapters, rank
        self.scale = torch.full((adapters,), 2.0, device=dev)
        self.codes, self.alpha = [], []
        for _ in range(depth):
            W = _inputs.normal((width, width), 1.2, g).to(dev)
            codes, alpha = tbn_quantize_pack(W)
            assert codes.shape[1] == packed_words(width)
            self.codes.append(codes)
            # the quantizer's grid is made for weights of about one; a block
            # of this width takes them at 1 / sqrt(width)
            self.alpha.append(alpha * width ** -0.5)
        # fp32 parameters by block: gamma, beta, a, b; b starts at zero, so
        # that an adapter changes nothing until it has learnt
        self.params = []
        for _ in range(depth):
            a = torch.randn((adapters, rank, width), generator=g).to(dev) * width ** -0.5
            self.params += [torch.ones(width, device=dev), torch.zeros(width, device=dev), a,
                            torch.zeros((adapters, rank, width), device=dev)]
        # the bf16 adapters that the kernels read; norm weights are read as fp32
        self.copies = [p.to(torch.bfloat16) if p.dim() == 3 else None for p in self.params]
        self.grads = [torch.zeros_like(p) for p in self.params]
        m, v, ms, vs = [], [], [], []
        for p in self.params:
            state = (AdamWPlan.state8(p) if p.dim() == 3 else
                     (torch.zeros_like(p), torch.zeros_like(p), None, None))
            for held, s in zip((m, v, ms, vs), state):
                held.append(s)
        self.plan = AdamWPlan(self.params, self.grads, m, v, ms, vs, copies=self.copies)
        self.steps = 0
        self._workspace = torch.empty(256, dtype=torch.uint8, device=dev)
        self._saved = None

    def _scratch(self, tokens: int, backward: bool) -> torch.Tensor:
        n = tbn_adapter_workspace_bytes(tokens, self.width, self.width, self.n, self.r, backward)
        if self._workspace.numel() < n:
            self._workspace = torch.empty(n, dtype=torch.uint8, device=self._workspace.device)
        return self._workspace

    def forward(self, x: torch.Tensor, ids: torch.Tensor, train: bool = True) -> torch.Tensor:
        """x [tokens, width] bf16 -> [tokens, width] bf16."""
        ws = self._scratch(x.shape[0], False)
        saved = []
        for l in range(self.depth):
            gamma, beta = self.params[4 * l:4 * l + 2]
            a, b = self.copies[4 * l + 2:4 * l + 4]
            h, mean, rstd = tbn_layernorm_fwd(x, gamma, beta)
            y = tbn_linear_fwd(h, self.codes[l], self.alpha[l], self.width, residual=x)
            v = torch.empty((x.shape[0], self.r), device=x.device) if train else None
            tbn_adapter_fwd(h, a, b, ids, self.scale, base=y, out=y, v=v, workspace=ws)
            saved.append((x, h, mean, rstd, v))
            x = y
        self._saved = (saved, ids) if train else None
        return x

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """dy [tokens, width] bf16, the loss's gradient at the last forward's
        result -> its gradient at x; the parameters' go to ``grads``."""
        saved, ids = self._saved
        tokens, width = dy.shape
        ws = self._scratch(tokens, True)
        for l in reversed(range(self.depth)):
            x, h, mean, rstd, v = saved[l]
            a, b = self.copies[4 * l + 2:4 * l + 4]
            dgamma, dbeta, da, db = self.grads[4 * l:4 * l + 4]
            # through the two-bit projection, as a 1x1 convolution over tokens
            dh = tbn_conv2d_bwd_data(dy.view(tokens, 1, 1, width), self.codes[l], self.alpha[l],
                                     width, (1, 1), 1, 1).view(tokens, width)
            tbn_adapter_bwd(dy, h, a, b, ids, self.scale, v=v, base=dh, dx=dh, da=da, db=db,
                            workspace=ws)
            dy, _, _ = tbn_layernorm_bwd(dh, x, mean, rstd, self.params[4 * l], dres=dy,
                                         dgamma=dgamma, dbeta=dbeta)
        return dy

    def step(self, lr: float) -> None:
        """One AdamW step of every adapter and norm weight with ``grads``."""
        self.steps += 1
        tbn_adamw_step(self.plan, self.steps, lr, seed=self.steps)


def main(argv=None) -> list:
    ap = argparse.ArgumentParser(description="fine-tune adapters of a two-bit network")
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--depth", type=int, default=4)
    ap.add_argument("--adapters", type=int, default=8)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--lr", type=float, default=2e-3)
    o = ap.parse_args(argv)
    g = _inputs.generator(1)
    net = AdaptedStack(o.width, o.depth, o.adapters, o.rank)
    x = torch.randn((o.tokens, o.width), generator=g).to(torch.bfloat16).cuda()
    ids = torch.randint(-1, o.adapters, (o.tokens,), generator=g, dtype=torch.int32).cuda()
    # what each adapter has to learn: its own offset of the frozen network's output
    offset = torch.randn((o.adapters + 1, o.width), generator=g).cuda()
    offset[-1] = 0
    target = net.forward(x, ids, train=False).float() + offset[ids.long()]
    losses = []
    for _ in range(o.steps):
        diff = net.forward(x, ids).float() - target
        losses.append(float((diff * diff).mean()))
        # the factor that makes this the gradient of the mean is left to
        # AdamW, which is free of scale
        net.backward(diff.to(torch.bfloat16))
        net.step(o.lr)
        if len(losses) % 10 == 1 or len(losses) == o.steps:
            print("step %3d  loss %.4f" % (len(losses), losses[-1]))
    served = torch.cat([net.forward(x[t:t + 1], ids[t:t + 1], train=False) for t in range(4)])
    error = float((served.float() - target[:4]).square().mean())
    print("served one token at a time: loss %.4f" % error)
    return losses + [error]


if __name__ == "__main__":
    main()
