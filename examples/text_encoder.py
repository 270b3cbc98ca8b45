"""A text encoder block that learns from its own alignment, and its streaming form.

Training, one step (`Encoder.step`): tokens become queries, keys and values; norm
and rotation of queries and keys (mas_qk_norm_rope); attention in which nearer
tokens count more (mas_attention); mu and log_sigma of every token; the
log-likelihoods of the frames (mas_loglik), their alignment (mas_search), and the
loss of the aligned frames with its gradients (mas_align_loss), which go back
through mas_attention_backward and mas_qk_norm_rope_backward to every weight.

Streaming (`Encoder.stream`): a causal pass token by token over a cache, where each
new key is written to its place by the norm's own call.

    python examples/text_encoder.py --steps 30
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2409_07704_amd as mas  # noqa: E402


class Encoder:
    """One attention block of `Hq` query and `Hk` key heads of `D` channels on
    `width` channels, in `dtype`, with fp32 outputs mu and log_sigma of `mel`
    channels; weights are fp32 in `self.w`."""

    def __init__(self, vocabulary=40, width=192, Hq=4, Hk=2, D=48, mel=80, longest=512, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator().manual_seed(seed)
        r = lambda *s: (torch.randn(s, generator=gen) / math.sqrt(s[0])).cuda()
        self.Hq, self.Hk, self.D, self.mel, self.dtype = Hq, Hk, D, mel, dtype
        self.w = {"embed": r(vocabulary, width) * math.sqrt(vocabulary), "qkv": r(width, (Hq + 2 * Hk) * D), "out": r(Hq * D, width),
                  "mu": r(width, mel), "log_sigma": 0.1 * r(width, mel), "q_gain": torch.ones(D, device="cuda"),
                  "k_gain": torch.ones(D, device="cuda")}
        angle = torch.arange(longest, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))
        self.cos, self.sin = torch.cos(angle).float().cuda(), torch.sin(angle).float().cuda()
        self.slope = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device="cuda")

    def heads(self, x):
        """Queries, keys and values of embedded tokens [B, T, width]: slices of one projection."""
        Hq, Hk = self.Hq, self.Hk
        qkv = (x.to(self.dtype) @ self.w["qkv"].to(self.dtype)).view(*x.shape[:2], Hq + 2 * Hk, self.D)
        return qkv[:, :, :Hq], qkv[:, :, Hq : Hq + Hk], qkv[:, :, Hq + Hk :]

    def forward(self, tokens, t_x):
        """mu, log_sigma [B, T, mel], and what the backward pass needs."""
        w, rest = self.w, (self.w["q_gain"], self.w["k_gain"], self.cos, self.sin)
        x = w["embed"][tokens]
        q0, k0, v = self.heads(x)
        q, k = mas.mas_qk_norm_rope(q0, k0, *rest, t_x=t_x)
        lse = torch.empty((x.shape[0], self.Hq, x.shape[1]), device="cuda")
        o = mas.mas_attention(q, k, v, t_q=t_x, t_k=t_x, slope=self.slope, lse_out=lse)
        y = x + (o.flatten(2) @ w["out"].to(self.dtype)).float()
        return y @ w["mu"], y @ w["log_sigma"], (tokens, t_x, x, q0, k0, q, k, v, o, lse, y)

    def backward(self, kept, dmu, dls):
        """Gradients of all weights from those of mu and log_sigma."""
        tokens, t_x, x, q0, k0, q, k, v, o, lse, y = kept
        w, B, T = self.w, *tokens.shape
        flat = lambda a: a.reshape(B * T, -1)
        g = {"mu": flat(y).T @ flat(dmu), "log_sigma": flat(y).T @ flat(dls)}
        dy = dmu @ w["mu"].T + dls @ w["log_sigma"].T
        dy16 = dy.to(self.dtype)
        g["out"] = flat(o).float().T @ flat(dy)
        do = (dy16 @ w["out"].T.to(self.dtype)).view_as(o)
        dqkv = torch.empty((B, T, self.Hq + 2 * self.Hk, self.D), dtype=self.dtype, device="cuda")
        dq, dk, dv = dqkv[:, :, : self.Hq], dqkv[:, :, self.Hq : self.Hq + self.Hk], dqkv[:, :, self.Hq + self.Hk :]
        mas.mas_attention_backward(do, q, k, v, o, lse, t_q=t_x, t_k=t_x, slope=self.slope, dq=dq, dk=dk, dv=dv)
        # The norm's gradients take the place of those they come from.
        _, _, g["q_gain"], g["k_gain"] = mas.mas_qk_norm_rope_backward(
            dq, dk, q0, k0, w["q_gain"], w["k_gain"], self.cos, self.sin, t_x=t_x, dq=dq, dk=dk)
        g["qkv"] = flat(x).T @ flat(dqkv).float()
        dx = dy + (flat(dqkv) @ w["qkv"].T.to(self.dtype)).view_as(dy).float()
        g["embed"] = torch.zeros_like(w["embed"]).index_add_(0, tokens.view(-1), flat(dx))
        return g

    def align(self, mu, log_sigma, z, t_x, t_y):
        """The best alignment of the frames under the tokens' Gaussians."""
        return mas.mas_search(mas.mas_loglik(mu, log_sigma, z, t_x, t_y), t_x, t_y)

    def step(self, tokens, z, t_x, t_y, rate=0.0):
        """One training step; the mean loss of a frame and channel, the weights'
        gradients and the alignment."""
        mu, log_sigma, kept = self.forward(tokens, t_x)
        row_start = self.align(mu, log_sigma, z, t_x, t_y)
        share = torch.full((len(tokens),), 1.0, device="cuda") / (t_y.sum() * self.mel)
        loss, dmu, dls, _ = mas.mas_align_loss(mu, log_sigma, z, row_start, item_weight=share)
        grads = self.backward(kept, dmu, dls)
        for n, g in grads.items():
            self.w[n] -= rate * g
        return (loss * share).sum(), grads, row_start

    def stream(self, tokens):
        """Causal attention of whole items, token by token over a cache: [B, T, Hq, D]."""
        B, T = tokens.shape
        cache_k, cache_v = (torch.zeros((B, T, self.Hk, self.D), dtype=self.dtype, device="cuda") for _ in range(2))
        out = torch.empty((B, T, self.Hq, self.D), dtype=self.dtype, device="cuda")
        for t in range(T):
            q, k, v = self.heads(self.w["embed"][tokens[:, t : t + 1]])
            pos, length = (torch.full(s, n, dtype=torch.int32, device="cuda") for s, n in (((B, 1), t), ((B,), t + 1)))
            q, _ = mas.mas_qk_norm_rope(q, k, self.w["q_gain"], self.w["k_gain"], self.cos, self.sin, pos=pos, k_out=cache_k[:, t : t + 1])
            cache_v[:, t : t + 1] = v
            mas.mas_attention(q, cache_k, cache_v, t_k=length, causal=True, slope=self.slope, out=out[:, t : t + 1])
        return out


def batch(B=8, T=60, S=240, mel=80, vocabulary=40, seed=1):
    """Tokens and frames that say them: every token sounds like itself, for a random
    number of frames."""
    gen = torch.Generator().manual_seed(seed)
    sound = torch.randn((vocabulary, mel), generator=gen)
    tokens = torch.randint(0, vocabulary, (B, T), generator=gen)
    t_x = torch.randint(T // 2, T + 1, (B,), generator=gen)
    t_y = torch.tensor([int(torch.randint(2 * int(n), S + 1, (1,), generator=gen)) for n in t_x])
    z = torch.randn((B, S, mel), generator=gen) * 0.3
    for b in range(B):
        cuts = torch.sort(torch.randperm(int(t_y[b]) - 1, generator=gen)[: int(t_x[b]) - 1] + 1).values
        row = torch.searchsorted(cuts, torch.arange(int(t_y[b])), right=True)
        z[b, : int(t_y[b])] += sound[tokens[b, row]]
    return tokens.cuda(), z.cuda(), t_x.to(torch.int32).cuda(), t_y.to(torch.int32).cuda()


def main(steps=30, rate=1.0):
    encoder, data = Encoder(), batch()
    losses = []
    for n in range(steps):
        loss = encoder.step(*data, rate=rate)[0]
        losses.append(loss.item())
        if n % 10 == 0 or n == steps - 1:
            print(f"step {n}: {losses[-1]:.4f} nats a frame and channel", flush=True)
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--steps", type=int, default=30)
    main(parser.parse_args().steps)
