"""The operators run together (examples/text_encoder.py): a training step against
automatic differentiation of the same step in 64 bits, a loss that falls, and a
causal pass token by token against the whole one."""
from __future__ import annotations

import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("text_encoder", os.path.join(ROOT, "examples", "text_encoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _reference(enc, tokens, z, t_x, t_y, row_start):
    """Loss and weights' gradients in 64 bits on the host, for a given alignment."""
    w = {n: x.cpu().double().requires_grad_() for n, x in enc.w.items()}
    tokens, z, row_start = tokens.cpu(), z.cpu().double(), row_start.cpu().long()
    cos, sin, slope = (x.cpu().double() for x in (enc.cos, enc.sin, enc.slope))
    Hq, Hk, D = enc.Hq, enc.Hk, enc.D
    total, frames = 0.0, int(t_y.sum())
    for b in range(len(tokens)):
        n = int(t_x[b])
        x = w["embed"][tokens[b, :n]]
        qkv = (x @ w["qkv"]).view(n, Hq + 2 * Hk, D)

        def turned(y, gain):
            y = y / torch.sqrt(y.square().mean(2, keepdim=True) + 1e-6) * gain
            a, c = y[..., : D // 2], y[..., D // 2 :]
            cs, sn = cos[:n, None], sin[:n, None]
            return torch.cat([a * cs - c * sn, c * cs + a * sn], 2)

        q, k, v = turned(qkv[:, :Hq], w["q_gain"]), turned(qkv[:, Hq : Hq + Hk], w["k_gain"]), qkv[:, Hq + Hk :]
        far = (torch.arange(n)[:, None] - torch.arange(n)[None]).abs()
        heads = []
        for h in range(Hq):
            s = q[:, h] @ k[:, h * Hk // Hq].T / math.sqrt(D) - slope[h] * far
            heads.append(torch.softmax(s, 1) @ v[:, h * Hk // Hq])
        y = x + torch.cat(heads, 1) @ w["out"]
        held = row_start[b, 1 : n + 1] - row_start[b, :n]
        mu, ls = (torch.repeat_interleave(y @ w[m], held, 0) for m in ("mu", "log_sigma"))
        r = (z[b, : len(mu)] - mu) * torch.exp(-ls)
        total = total + (0.5 * math.log(2 * math.pi) + ls + 0.5 * r * r).sum()
    loss = total / (frames * enc.mel)
    return loss.detach(), dict(zip(w, torch.autograd.grad(loss, list(w.values()))))


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 0.03)])
def test_a_training_step(example, dtype, tol):
    """fp32: some hundred fp32 roundings on the way; bf16: activations rounded a
    handful of times at 2^-8 each, so a few percent of a gradient's norm at most."""
    enc, data = example.Encoder(dtype=dtype), example.batch()
    loss, grads, row_start = enc.step(*data)
    print(f"[gpu-case] training step {dtype}", flush=True)
    want, wgrads = _reference(enc, *data, row_start)
    assert abs(loss.item() - want.item()) <= tol * abs(want.item())
    for n, g in grads.items():
        off = (g.cpu().double() - wgrads[n]).norm() / wgrads[n].norm()
        assert off <= tol, (n, off.item())


def test_the_loss_falls(example):
    losses = example.main(steps=30)
    assert losses[-1] < losses[0] - 0.2 and all(math.isfinite(x) for x in losses)


def test_streaming_equals_the_whole_pass(example):
    import paper_2409_07704_amd as mas

    enc = example.Encoder(dtype=torch.float32)
    tokens = example.batch(B=3, T=37, S=100)[0]
    got = enc.stream(tokens)
    q, k, v = enc.heads(enc.w["embed"][tokens])
    q, k = mas.mas_qk_norm_rope(q, k, enc.w["q_gain"], enc.w["k_gain"], enc.cos, enc.sin)
    want = mas.mas_attention(q, k, v, causal=True, slope=enc.slope)
    # Two fp32 evaluations of averages of at most 37 values.
    assert float((got - want).abs().max()) <= 1e-5 * float(want.abs().max())
