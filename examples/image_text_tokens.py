"""Photos and text to the normalised rows of one sequence, forward, backward
and a few steps of gradient descent: the preprocessing and the token operators
as a fine-tuning loop uses them.

    python examples/image_text_tokens.py [--steps N]

Every step takes a ragged batch of photos through the preprocessing (uint8 to
fp16, NCHW), projects their 16 x 16 patches into rows 1 .. 196 of a bf16
sequence, looks the other rows up by token id, and normalises all of them. The
loss pulls the normalised rows towards fixed random ones, so that every
parameter has a gradient: projection, bias, positions, table, norm weights.
Parameters are kept in fp32 and used in bf16; all buffers are made once.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2007_13005_amd import smol, synthetic, tokens  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
PATCH, SIDE, DIM, VOCAB, TEXT = 16, 224, 384, 1000, 31


class Front:
    """The parameters (fp32 masters, bf16 copies), gradients and buffers."""

    def __init__(self, wl, device, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        rows = (SIDE // PATCH) ** 2
        length = 1 + rows + TEXT

        def new(*shape, scale):
            return (torch.randn(shape, generator=g) * scale).to(device)

        self.params = {"weight": new(DIM, 3, PATCH, PATCH, scale=0.03), "bias": new(DIM, scale=0.1),
                       "pos": new(rows, DIM, scale=0.1), "table": new(VOCAB, DIM, scale=0.03),
                       "gamma": 1 + new(DIM, scale=0.1), "beta": new(DIM, scale=0.1)}
        self.low = {k: v.to(BF16) for k, v in self.params.items()}
        self.grads = {k: torch.empty_like(v) for k, v in self.params.items()}
        n = wl.n
        ids = torch.randint(0, VOCAB, (n, length), generator=g)
        ids[:, 1:1 + rows] = -1  # the places of the image's rows
        self.ids = ids.to(device)
        self.target = new(n, length, DIM, scale=1.0)
        self.rows, self.scale = rows, DIM ** 0.5
        self.images = torch.empty((n, 3, SIDE, SIDE), dtype=torch.float16, device=device)
        self.seq = torch.empty((n, length, DIM), dtype=BF16, device=device)
        self.out, self.grad = torch.empty_like(self.seq), torch.empty_like(self.seq)
        self.mean = torch.empty((n, length), dtype=F32, device=device)
        self.rstd = torch.empty_like(self.mean)
        need = max(tokens.layer_norm_workspace_bytes(n * length, DIM),
                   tokens.embed_workspace_bytes(n * length, VOCAB, DIM),
                   tokens.patch_embed_workspace_bytes(self.images, self.grads["weight"], BF16))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    def step(self, wl, src, rate: float) -> torch.Tensor:
        """One step of gradient descent; the loss before it, on the device."""
        p, g, image_rows = self.low, self.grads, self.seq[:, 1:1 + self.rows]
        smol.preprocess_batch(src, wl.offsets, wl.widths, wl.heights, smol.make_params(
            256, SIDE, SIDE, wl.mean, wl.std, smol.OUT_F16), out=self.images)
        tokens.embed(self.ids, p["table"], self.scale, out=self.seq, keep=True)
        tokens.patch_embed(self.images, p["weight"], p["bias"], p["pos"], out=image_rows)
        tokens.layer_norm(self.seq, self.params["gamma"], self.params["beta"], out=self.out,
                          mean=self.mean, rstd=self.rstd)
        off = self.out.float() - self.target
        loss = (off * off).mean()
        grad_out = (off * (2.0 / DIM)).to(BF16)  # of the loss's sum over rows
        tokens.layer_norm_backward(grad_out, self.seq, self.params["gamma"], self.mean, self.rstd,
                                   self.grad, g["gamma"], g["beta"], workspace=self.workspace)
        tokens.patch_embed_backward(self.grad[:, 1:1 + self.rows], self.images, g["weight"],
                                    g["bias"], g["pos"], workspace=self.workspace)
        tokens.embed_backward(self.grad, self.ids, g["table"], self.scale,
                              workspace=self.workspace)
        for k, v in self.params.items():
            v.add_(g[k], alpha=-rate)
            self.low[k].copy_(v)
        return loss


# The sum of squares' curvature along the projection is about rows * values * 2
# / dim = 8 * 196 * 768 * 2 / 384 (inputs and 1 / rstd about 1): steps below
# 2 / 6300 descend.
RATE = 1e-4


def run(steps: int = 20, photos: int = 8, rate: float = RATE) -> list[float]:
    wl = synthetic.c2(n=photos)
    src = torch.from_numpy(wl.src).to("cuda")
    front = Front(wl, "cuda")
    return [float(loss) for loss in [front.step(wl, src, rate) for _ in range(steps)]]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=20)
    losses = run(ap.parse_args().steps)
    for i, loss in enumerate(losses):
        print(f"step {i}: loss {loss:.4f}", flush=True)
