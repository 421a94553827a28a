"""A linear map with 4-bit weights: trained from 8-bit saved batches, then served by coded workers.

Training, each step:
  the batch is saved in 8 bits (coded_mx_quantize), which is all that is kept of it;
  Y = X W^T - T from the saved batch and the 4-bit weights (coded_mx_mm, C = T);
  dW = Y^T X from the saved batch (coded_mx_mm_t) and dX = Y W (coded_mx_mm_t), what a layer before would get;
  the fp32 master weights move against dW and are stored in 4 bits again.

Serving: the systematic workers of an (n, k) code hold block rows of the codes as they lie and multiply by them
(coded_mx_mm); the parity workers hold coded blocks of the same values (coded_encode, coded_worker_mm); the result is
decoded from any k of the n (coded_decode).

  python examples/mx_linear.py [--tokens 4096 --features 1024 --outputs 1500 --steps 30]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synth  # noqa: E402
from paper_1512_02673_amd import binding as lib  # noqa: E402


def train(tokens: int, features: int, outputs: int, steps: int, rate: float = 0.5, seed: int = 0):
    """(losses, 4-bit weights, gradient of the last batch) of `steps` steps towards a random map."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    target = torch.randn((outputs, features), generator=g, device="cuda") / features ** 0.5
    master = torch.zeros_like(target)
    weights = lib.alloc_mx(outputs, features, lib.CODED_MX4)
    saved = lib.alloc_mx(tokens, features, lib.CODED_MX8)
    diff = torch.empty((tokens, outputs), dtype=torch.bfloat16, device="cuda")
    d_weights = torch.empty_like(master)
    d_batch = torch.empty((tokens, features), dtype=torch.bfloat16, device="cuda")
    losses = []
    for _ in range(steps):
        batch = torch.randn((tokens, features), generator=g, device="cuda").to(torch.bfloat16)
        wanted = (batch.float() @ target.t()).to(torch.bfloat16)
        lib.coded_mx_quantize(master, weights)
        lib.coded_mx_quantize(batch, saved)
        del batch
        lib.coded_mx_mm(weights, saved, diff, x_rows=True, y_rows=True, beta=-1.0, C=wanted)
        losses.append(diff.float().square().mean())
        lib.coded_mx_mm_t(saved, diff, d_weights, y_rows=True, alpha=1.0 / tokens)
        lib.coded_mx_mm_t(weights, diff, d_batch, x_rows=True, y_rows=True)
        master -= rate * d_weights
    lib.coded_mx_quantize(master, weights)
    return torch.stack(losses).tolist(), weights, d_batch


def serve(weights: "lib.MXMatrix", x: torch.Tensor, n: int, k: int, seed: int = 0, draw: int = 0):
    """(decoded result, survivors, info) of the coded product of the weights with x (features x s, bf16)."""
    q, r = weights.shape
    s = x.shape[1]
    code = lib.Code.systematic(synth.parity_matrix(n, k, seed, dtype="bf16"), 2)
    qb = code.qb(q)
    # once per set of weights: the parity workers' blocks, from the values the codes stand for
    values = torch.empty((q, r), dtype=torch.bfloat16, device=x.device)
    lib.coded_mx_dequantize(weights, values)
    parity = lib.alloc_parity(code, q, r, torch.bfloat16)
    lib.coded_encode(code, values, parity)
    # per x: the systematic workers' block rows are consecutive, so one product over the codes serves all of them
    results = lib.alloc_y(code, q, s, torch.float32)
    systematic = results[:k].view(k * qb, s)
    systematic[q:].zero_()
    lib.coded_mx_mm(weights, x, systematic[:q])
    mask = np.zeros(n, dtype=np.uint8)
    mask[k:] = 1
    lib.coded_worker_mm(code, values, parity, x, results, worker_mask=mask)
    survivors, _ = lib.coded_draw_survivors(n, k, seed, draw)
    for w in set(range(n)) - set(int(w) for w in survivors):
        results[w].fill_(float("nan"))   # these never arrive
    out = torch.empty((q, s), dtype=torch.float32, device=x.device)
    info = torch.zeros(1, dtype=torch.int32, device=x.device)
    lib.coded_decode(code, survivors, results, q, out, info)
    return out, survivors, info


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--features", type=int, default=1024)
    p.add_argument("--outputs", type=int, default=1500)
    p.add_argument("--steps", type=int, default=30)
    a = p.parse_args()
    losses, weights, _ = train(a.tokens, a.features, a.outputs, a.steps)
    print("mean squared error by step: " + " ".join(f"{v:.4f}" for v in losses[:: max(1, a.steps // 10)]) + f" ... {losses[-1]:.4f}")
    x = torch.randn((a.features, 1), device="cuda").to(torch.bfloat16)
    plain = torch.empty((a.outputs, 1), dtype=torch.float32, device="cuda")
    lib.coded_mx_mm(weights, x, plain)
    for draw in range(3):
        out, survivors, info = serve(weights, x, 16, 12, seed=2, draw=draw)
        missing = sorted(set(range(12)) - set(survivors.tolist()))
        err = float((out - plain).norm() / plain.norm())
        print(f"(16,12) coded product, blocks {missing} decoded from parity: {err:.2e} from the plain one, info {int(info.item())}")


if __name__ == "__main__":
    main()
