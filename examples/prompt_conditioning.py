"""A video diffusion transformer's prompt path, trained for a few steps and then
used for one denoising step.

    python examples/prompt_conditioning.py [--steps 20] [--tokens 1984] [--prompt 64]

A text encoder layer (self-attention with a learned relative position bias)
turns prompts of different lengths into states; the video tokens read them by
cross attention.  Both run forward and backward in the library's kernels; the
guided and the unguided sample of a pair go side by side, the unguided one with
an empty prompt.  The denoising step then runs the block's own attention
through the search schedule and reads the prompt once.
"""
import argparse
import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2502_21079_amd as ad  # noqa: E402
from paper_2502_21079_amd.schedule import AdaSpaAttention, SearchSchedule  # noqa: E402


class PromptEncoderLayer(nn.Module):
    """Self-attention over a prompt; scores get a learned value per head and
    distance bucket and no scaling."""

    def __init__(self, width, heads, buckets=32, max_distance=128):
        super().__init__()
        self.heads, self.max_distance = heads, max_distance
        self.norm = nn.LayerNorm(width)
        self.qkv = nn.Linear(width, 3 * width, bias=False)
        self.proj = nn.Linear(width, width, bias=False)
        self.table = nn.Parameter(torch.zeros(buckets, heads))
        with torch.no_grad():
            self.qkv.weight[:width] *= (width // heads) ** -0.5

    def forward(self, x, lens):
        B, L, W = x.shape
        q, k, v = self.qkv(self.norm(x)).view(B, L, 3, self.heads, -1).permute(2, 0, 3, 1, 4)
        y = ad.rel_bias_attention(q, k, v, self.table, max_distance=self.max_distance, key_lens=lens, scale=1.0)
        return x + self.proj(y.transpose(1, 2).reshape(B, L, W))


class ReadPrompt(nn.Module):
    """Video tokens read the prompt's states."""

    def __init__(self, width, heads):
        super().__init__()
        self.heads = heads
        self.norm = nn.LayerNorm(width)
        self.q = nn.Linear(width, width, bias=False)
        self.kv = nn.Linear(width, 2 * width, bias=False)
        self.proj = nn.Linear(width, width, bias=False)

    def forward(self, x, states, lens):
        B, L, W = x.shape
        q = self.q(self.norm(x)).view(B, L, self.heads, -1).transpose(1, 2)
        k, v = self.kv(states).view(B, -1, 2, self.heads, W // self.heads).permute(2, 0, 3, 1, 4)
        y = ad.cross_attention(q, k, v, key_lens=lens)
        return x + self.proj(y.transpose(1, 2).reshape(B, L, W))


def run(steps=20, tokens=1984, prompt=64, heads=2, head_dim=64, seed=0, device="cuda"):
    """Trains the two layers and runs one denoising step; returns the losses and
    the step's output."""
    torch.manual_seed(seed)
    width, dt = heads * head_dim, torch.bfloat16
    encode = PromptEncoderLayer(width, heads).to(device, dt)
    read = ReadPrompt(width, heads).to(device, dt)
    words = torch.randn(2, prompt, width, device=device).to(dt)
    lens = torch.tensor([prompt, 0], dtype=torch.int32, device=device)    # with and without the prompt
    video = torch.randn(1, tokens, width, device=device).expand(2, -1, -1).to(dt)
    # What the guided sample should become: the video tokens moved towards the
    # first word; the unguided one stays as it is.
    want = torch.stack((video[0] + 0.5 * words[0, 0], video[1])).detach()

    params = [*encode.parameters(), *read.parameters()]
    opt = torch.optim.AdamW(params, lr=2e-3, weight_decay=0.0)
    losses = []
    for _ in range(steps):
        y = read(video, encode(words, lens), lens)
        loss = (y.float() - want.float()).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))

    # One block of one denoising step: the video's own attention (searched),
    # then the prompt.
    own = AdaSpaAttention((2, heads, tokens, head_dim), block=64, text_start=0, text_len=0, mode="topk",
                          head_param_bp=[5000] * heads, schedule=SearchSchedule((0,)), device=device)
    with torch.no_grad():
        x = video.reshape(2, tokens, heads, head_dim).transpose(1, 2).contiguous()
        y, _ = own.step(0, x, x, x)
        x = video + y.transpose(1, 2).reshape(2, tokens, width)
        out = read(x, encode(words, lens), lens)
    return losses, x, out


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=1984)
    ap.add_argument("--prompt", type=int, default=64)
    a = ap.parse_args()
    losses, before, out = run(a.steps, a.tokens, a.prompt)
    print("loss %.4f -> %.4f over %d steps" % (losses[0], losses[-1], len(losses)))
    moved = (out.float() - before.float()).abs().mean((1, 2)).tolist()
    print("the prompt moves the guided sample by %.3f, the unguided one by %.3f" % tuple(moved))


if __name__ == "__main__":
    main()
