"""A small classifier of long byte sequences, trained on a synthetic task: `python -m paper_2302_06646_amd.classifier [--steps 60]`.

One long-convolution block and what stands around it, every step of it a call of this library (torch owns the memory, transposes,
and computes the head and its loss):

    x0   = dropout(sqrt(H) E[tokens])                       longconv_embed_fwd, straight into [B, H, N]
    kbar = Squash(Smooth(dropout(K)))                       longconv_kreg_fwd_seeded
    x1   = x0 + dropout((x0 * kbar)[:N] + D x0)             longconv_fwd, longconv_dropout_fwd with one value for each row
    z    = silu(group norm(x1 transposed))                  longconv_gnorm_fwd, [B, N, H]
    logits = mean over the sequence's places of z, times the head

With `--mixer scan` the block of selective.py stands in the convolution's place: x1 = x0 + dropout(selective(x0)), up to each sequence's end.

No mask is stored: the backward pass draws each of them again from (seed, number of the call).  Sequences are of uneven lengths; their
padding is token -1, which embeds to zeros and has no gradient.

The task: in a sequence of random bytes, one of the first `classes` bytes comes up more often than the others; which?
"""
from __future__ import annotations

import argparse
import math

import torch

import paper_2302_06646_amd as lc
from paper_2302_06646_amd.selective import Selective

VOCABULARY = 256


class Classifier:
    """Parameters (fp32, float32 gradients in `.grad`), workspaces and activations for batches of B sequences of N tokens."""

    def __init__(self, B, N, H=64, classes=4, groups=8, dtype=torch.bfloat16, drop=0.1, kernel_drop=0.2, tied_drop=0.1, seed=0,
                 mixer="conv"):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.B, self.N, self.H, self.groups, self.seed = B, N, H, groups, seed
        self.drop, self.kernel_drop, self.tied_drop = drop, kernel_drop, tied_drop
        self.scale, self.eps, self.width, self.squash = math.sqrt(H), 1e-5, 1, 1e-3
        decay = torch.exp(-4.0 * torch.arange(N, device="cuda") / N)
        self.p = {"E": randn(VOCABULARY, H) / math.sqrt(H), "K": randn(H, N) / math.sqrt(N) * decay, "D": randn(H),
                  "gamma": torch.ones(H, device="cuda"), "beta": torch.zeros(H, device="cuda"),
                  "head": (randn(H, classes) / math.sqrt(H))}
        self.block = None
        if mixer == "scan":
            del self.p["K"], self.p["D"]
            self.block = Selective(B, N, H, dtype=dtype, generator=g)
        elif mixer != "conv":
            raise ValueError(f"mixer: expected conv or scan, got {mixer}")
        for t in self.p.values():
            t.grad = torch.zeros_like(t)
        if self.block:
            self.p.update(self.block.p)
        io = lc.dtype_code(torch.empty(0, dtype=dtype))
        new = lambda *s, dt=dtype: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        self.x0, self.y, self.x1, self.dx1, self.dy, self.dx0 = (new(B, H, N) for _ in range(6))
        self.z, self.dt = new(B, N, H), new(B, N, H)
        if mixer == "conv":
            self.kbar, self.dkbar = torch.empty_like(self.p["K"]), torch.empty_like(self.p["K"])
            self.ws = lc.new_workspace(B, H, N, io, True)
        self.mean, self.rstd = (new(B, groups, dt=torch.float32) for _ in range(2))
        self.ws_embed = lc.new_workspace_embed(B, N, VOCABULARY, H, io, lc.CHANNELS_FIRST)
        self.ws_gnorm = lc.new_workspace_gnorm(B, N, H, groups, io, True)
        lc.longconv_init()

    def forward(self, tokens, step):
        """Logits [B, classes] of tokens [B, N]; `step` numbers the training steps, and with them the masks."""
        p, call = self.p, 3 * step
        lc.longconv_embed_fwd(tokens, p["E"], self.x0, self.scale, lc.CHANNELS_FIRST, self.drop, self.seed, call)
        if self.block:
            self.lengths = (tokens >= 0).sum(1)               # (a sequence's padding is behind its end)
            self.block.refresh()
            self.block.forward(self.x0, self.y, self.lengths)
        else:
            lc.longconv_kreg_fwd_seeded(p["K"], self.kbar, self.width, self.squash, self.kernel_drop, self.seed, call + 1)
            lc.longconv_fwd(self.x0, self.kbar, p["D"], self.y, self.ws)
        lc.longconv_dropout_fwd(self.y, self.x1, self.tied_drop, self.seed, call + 2, residual=self.x0, tie=self.N)
        self.t = self.x1.transpose(1, 2).contiguous()
        lc.longconv_gnorm_fwd(self.t, p["gamma"], p["beta"], self.z, self.mean, self.rstd, self.eps, "silu", self.ws_gnorm)
        self.there = (tokens >= 0).float() / (tokens >= 0).sum(1, keepdim=True).clamp(min=1)      # (none: nothing is pooled)
        self.pooled = (self.z.float() * self.there[..., None]).sum(1)
        return self.pooled @ p["head"]

    def backward(self, dlogits, tokens, step):
        """Gradients of all parameters from those of the logits; after forward() of the same tokens and step."""
        p, call = self.p, 3 * step
        p["head"].grad.copy_(self.pooled.t() @ dlogits)
        dz = ((dlogits @ p["head"].t())[:, None, :] * self.there[..., None]).to(self.z.dtype)
        lc.longconv_gnorm_bwd(dz, self.t, p["gamma"], p["beta"], self.mean, self.rstd, self.dt, p["gamma"].grad, p["beta"].grad, "silu",
                              self.ws_gnorm)
        self.dx1.copy_(self.dt.transpose(1, 2))
        lc.longconv_dropout_bwd(self.dx1, self.dy, self.tied_drop, self.seed, call + 2, tie=self.N)
        if self.block:
            self.block.backward(self.dy, self.x0, self.dx0, self.lengths)
        else:
            lc.longconv_bwd(self.dy, self.x0, self.kbar, p["D"], self.dx0, self.dkbar, p["D"].grad, self.ws)
            lc.longconv_kreg_bwd_seeded(p["K"], self.dkbar, p["K"].grad, self.width, self.squash, self.kernel_drop, self.seed, call + 1)
        self.dx0.add_(self.dx1)                               # the residual's gradient
        lc.longconv_embed_bwd(self.dx0, tokens, p["E"].grad, self.scale, lc.CHANNELS_FIRST, self.ws_embed, self.drop, self.seed, call)

    def step(self, tokens, labels, step, optimizer):
        """One training step; returns its loss and accuracy as tensors."""
        logits = self.forward(tokens, step)
        share = torch.softmax(logits, 1)
        target = torch.nn.functional.one_hot(labels, logits.shape[1]).float()
        loss = -(torch.log_softmax(logits, 1) * target).sum(1).mean()
        self.backward((share - target) / len(labels), tokens, step)
        optimizer.step()
        return loss, (logits.argmax(1) == labels).float().mean()


def batch(B, N, classes, generator):
    """Tokens [B, N] (-1 behind each sequence's end) and labels [B] of the task."""
    rand = lambda *s: torch.rand(*s, generator=generator, device="cuda")  # noqa: E731
    labels = (rand(B) * classes).long()
    tokens = (rand(B, N) * VOCABULARY).long()
    tokens = torch.where(rand(B, N) < 0.05, labels[:, None], tokens)
    return torch.where(torch.arange(N, device="cuda") < (0.3 + 0.7 * rand(B, 1)) * N, tokens, -1), labels


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--length", type=int, default=2048, help="a power of two, 256 to 131072")
    ap.add_argument("--width", type=int, default=64)
    ap.add_argument("--mixer", choices=("conv", "scan"), default="conv")
    a = ap.parse_args(argv)
    model = Classifier(a.batch, a.length, a.width, mixer=a.mixer)
    optimizer = torch.optim.Adam(list(model.p.values()), lr=3e-3)
    generator = torch.Generator(device="cuda").manual_seed(1)
    for i in range(a.steps):
        loss, right = model.step(*batch(a.batch, a.length, 4, generator), i, optimizer)
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {loss.item():.4f}  accuracy {right.item():.2f}", flush=True)
    return loss.item()


if __name__ == "__main__":
    main()
