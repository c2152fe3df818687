"""Trains a stack of feed-forward blocks with M-FAC, with the activations kept whole or in 8 bits.

    python examples/feed_forward_mfac.py [--gated [--dropout P]] [--copy8] [--bf16] [--steps N] [--dim D] [--blocks B]
                                         [--rows R]

The task is regression onto a fixed random network of the same shape. Prints the
loss, the bytes that the forward pass keeps for the backward pass, and the time
of a step.
"""

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2107_03356_amd import nn  # noqa: E402
from paper_2107_03356_amd.optim import MFAC  # noqa: E402


def model(dim, blocks, copy8, device, gated=False, dropout=0.0):
    if gated:   # rms norms, gated layers, a learned gate for each channel
        return torch.nn.Sequential(nn.GatedStack(dim, 8 * dim // 3, blocks, gate=1.0, p=dropout, copy8=copy8, device=device),
                                   nn.Linear(dim, dim, device=device))
    return torch.nn.Sequential(*[nn.FeedForward(dim, 4 * dim, act="gelu_tanh", copy8=copy8, device=device)
                                 for _ in range(blocks)],
                               nn.LayerNorm(dim, copy8=copy8, device=device), nn.Linear(dim, dim, device=device))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--gated", action="store_true", help="gated blocks (GatedStack) in place of plain ones")
    ap.add_argument("--dropout", type=float, default=0.0, help="dropout of the gated blocks")
    ap.add_argument("--copy8", action="store_true", help="keep activations in 8 bits")
    ap.add_argument("--bf16", action="store_true", help="bfloat16 activations (parameters stay float32)")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--rows", type=int, default=4096)
    a = ap.parse_args()
    dev = torch.device("cuda:0")
    torch.manual_seed(0)
    dtype = torch.bfloat16 if a.bf16 else torch.float32
    x = torch.randn(a.rows, a.dim, device=dev)
    with torch.no_grad():
        target = model(a.dim, a.blocks, False, dev, a.gated)(x)
    x = x.to(dtype)
    net = model(a.dim, a.blocks, a.copy8, dev, a.gated, a.dropout)
    opt = MFAC(net.parameters(), lr=0.05, m=32, damp=1e-2)

    kept = {}

    def count(t):
        s = t.untyped_storage()   # parameters are there anyway
        if not any(s.data_ptr() == p.untyped_storage().data_ptr() for p in net.parameters()):
            kept[s.data_ptr()] = s.nbytes()
        return t

    for step in range(a.steps):
        opt.zero_grad()
        torch.cuda.synchronize()
        began = time.perf_counter()
        if step == 0:
            with torch.autograd.graph.saved_tensors_hooks(count, lambda t: t):
                y = net(x)
        else:
            y = net(x)
        loss = (y.float() - target).square().mean()
        loss.backward()
        opt.step()
        torch.cuda.synchronize()
        took = time.perf_counter() - began
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step:4d}  loss {loss.item():.5f}  {took * 1e3:.2f} ms", flush=True)
    print(f"kept for the backward pass: {sum(kept.values()) / 2 ** 20:.1f} MiB; optimizer status {opt.status()}")


if __name__ == "__main__":
    main()
