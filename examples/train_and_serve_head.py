"""Trains a small next-token model with Ember and serves it with an 8-bit head.

The model is an embedding, one residual addition with an RMS norm, and an LM
head, on a synthetic Markov chain: from each token one successor follows nine
times out of ten.  One training step is

    hidden, h = rmsnorm(embedding rows, gain, residual)    Ops.rmsnorm
    logits = hidden W^T                                    torch.matmul
    loss, dlogits = cross-entropy and its gradient         Ops.softmax_loss
    G = dlogits^T hidden                                   Ember.lmhead_grad
    dh, dgain = gradients of the norm                      Ops.rmsnorm_backward
    all gradients clipped by their global norm             Ops.clip_grads
    head, embedding, gain stepped                          Ember.step_dense, Ember.step_sparse

and serving one token for a batch of sequences is

    q, scales, _ = rmsnorm_quant(embedding rows, gain, residual)
    logits = matmul_quant(q, scales, wq, ws)               W once in 8 bits: Ops.quantize_rows

    python examples/train_and_serve_head.py [--steps N]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_01455_gb300 import Ember, Ops  # noqa: E402


def train_and_serve(steps=60, V=1024, D=256, T=2048, batch=16, tokens=32, max_norm=1.0, seed=0, device="cuda", say=print):
    """(first loss, last loss, share of generated tokens that are the chain's likely successor)."""
    g = torch.Generator(device=device).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=device)

    successor = torch.randperm(V, generator=g, device=device)
    E, W = (randn(V, D) * 0.5).bfloat16(), (randn(V, D) * 0.02).bfloat16()
    residual = (randn(1, D) * 0.1).bfloat16()
    gain = torch.ones(D, device=device)
    head = Ember(V, D, wdtype="bf16", device=device)
    embedding = Ember(V, D, wdtype="bf16", max_sparse_N=T, device=device)
    ops = Ops(device)
    G = torch.empty(V, D, device=device)
    first = last = None
    for t in range(1, steps + 1):
        ids = torch.randint(0, V, (T,), generator=g, device=device)
        noise = torch.randint(0, V, (T,), generator=g, device=device)
        likely = torch.rand(T, generator=g, device=device) < 0.9
        targets = torch.where(likely, successor[ids], noise)

        hidden, h = ops.rmsnorm(E[ids], gain, residual=residual.expand(T, D).contiguous())
        logits = hidden @ W.T
        loss, _, dlogits = ops.softmax_loss(logits, targets)
        dhidden = dlogits @ W
        dh, dgain = ops.rmsnorm_backward(dhidden, h, gain)
        head.lmhead_grad(dlogits, hidden, G)
        rows = dh.float()
        norm = ops.clip_grads([G, rows, dgain], max_norm)
        lr = 2e-2 * (1 - (t - 1) / steps)
        head.step_dense(W, G, lr, t)
        embedding.step_sparse(E, ids, rows, lr, t)
        gain -= lr * dgain
        if t == 1 or t == steps or t % 20 == 0:
            last = loss.item()
            first = last if first is None else first
            say(f"step {t}: loss {last:.3f}, gradient norm {norm.item():.3f}")

    wq, ws = ops.quantize_rows(W)
    ids = torch.randint(0, V, (batch,), generator=g, device=device)
    right = 0
    for _ in range(tokens):
        q, scales, _ = ops.rmsnorm_quant(E[ids], gain, residual=residual.expand(batch, D).contiguous())
        nxt = ops.matmul_quant(q, scales, wq, ws).argmax(1)
        right += int((nxt == successor[ids]).sum())
        ids = nxt
    assert ops.device_status() == 0 and head.device_status() == 0 and embedding.device_status() == 0
    share = right / (batch * tokens)
    say(f"8-bit head: {100 * share:.1f} % of {batch * tokens} generated tokens are the chain's likely successor")
    return first, last, share


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    train_and_serve(p.parse_args().steps)
