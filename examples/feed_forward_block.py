"""The feed-forward block of a diffusion transformer in 8 bits: quantize its weights once, run it,
capture it in a graph, and compare with the same block in binary32.

    python examples/feed_forward_block.py [tokens]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_33496_amd import cham, synth  # noqa: E402
from paper_2609_33496_amd.feed_forward import FeedForward  # noqa: E402


def main():
    tokens = int(sys.argv[1]) if len(sys.argv) > 1 else 8192
    d, hidden = 1152, 4608
    dev = torch.device("cuda:0")
    w_in, w_out = synth.hetero_weights_dev(1, hidden, d, dev), synth.hetero_weights_dev(2, d, hidden, dev)
    g = torch.ones(d, device=dev)
    x = synth.diffusion_acts_dev(3, 0, 300, tokens, d, dev).to(torch.bfloat16)
    r = synth.diffusion_acts_dev(3, 1, 300, tokens, d, dev)

    block = FeedForward(w_in, w_out, g, act=cham.ACT_GELU_TANH)
    y, h = block(x, r)

    n = torch.nn.functional.rms_norm(x.float() + r, (d,), g, 1e-6)
    want = torch.nn.functional.gelu(n @ w_in.t(), approximate="tanh") @ w_out.t()
    print(f"{tokens} tokens, {d} -> {hidden} -> {d}: relative difference from binary32 "
          f"{float((y.float() - want).norm() / want.norm()):.3f}")

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block(x, r)
    graph.replay()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(20):
        graph.replay()
    end.record()
    end.synchronize()
    us = begin.elapsed_time(end) / 20 * 1e3
    print(f"{us:.1f} us a pass in a graph, {4 * tokens * d * hidden / us / 1e6:.0f} TFLOP/s")


if __name__ == "__main__":
    main()
