"""A training step of a deep pre-norm stack, with and without 8-bit checkpoints.

Samples nodes of a 2-D domain, builds their radius graph, and runs the forward
and backward pass of a stack of message-passing layers between group norms both
ways: the time of a step, what it keeps from the forward to the backward pass,
and how far the gradients are from those of the full-precision activations.

    python examples/checkpointed_stack.py [--nodes 8192] [--layers 8] [--steps 5]
"""

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2402_15106_amd as dm  # noqa: E402


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--nodes", type=int, default=8192)
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=5)
    a = ap.parse_args()
    lib, dev = dm.Dsmp(0), torch.device("cuda", 0)
    torch.manual_seed(0)
    d, h, n = 64, 128, a.nodes
    pos = torch.rand(8 * n, 2, device=dev)
    pos = lib.dsmp_gather_rows(pos, lib.dsmp_sample_nodes(8 * n, n, 1))
    graph = lib.dsmp_radius_graph_build(pos, n, (40.0 / (3.1416 * n)) ** 0.5)
    attr = torch.cat([pos, torch.randn(n, 1, device=dev)], 1)
    x, gy = torch.randn(n, d, device=dev), torch.randn(n, d, device=dev)

    def uniform(*shape):
        return (2 * torch.rand(*shape, device=dev) - 1) * shape[-1] ** -0.5

    shapes = dm.StackShapes(n, 2, d, h, h, dm.BF16, a.layers, groups=8)
    norms = [(torch.ones(d, device=dev), torch.zeros(d, device=dev)) for _ in range(a.layers + 1)]
    results, packed = {}, None
    for checkpoints in (False, True):
        stack = dm.CheckpointedStack(lib, graph, shapes, checkpoints=checkpoints)
        if packed is None:
            packed = [lib.dsmp_nnconv_pack(stack.conv, {
                "W1": uniform(h, 6), "b1": uniform(h), "W2": uniform(h, h), "b2": uniform(h), "W3": uniform(d * d, h),
                "b3": uniform(d * d), "Wr": uniform(d, d), "br": uniform(d)}) for _ in range(a.layers)]
        for step in range(a.steps + 1):
            if step == 1:
                torch.cuda.synchronize()
                t = time.perf_counter()
            stack.forward(packed, norms, attr, x)
            grad_x, conv, norm = stack.backward(gy)
        torch.cuda.synchronize()
        ms = (time.perf_counter() - t) / max(1, a.steps) * 1e3
        results[checkpoints] = [grad_x] + [v for m in conv + norm for v in m.values()]
        print("%-20s %8.2f ms a step, %9.1f MB kept" % ("8-bit checkpoints" if checkpoints else "all activations", ms,
                                                        stack.kept_bytes() / 1e6))
        del stack
    far = max(float((u - v).double().norm() / v.double().norm()) for u, v in zip(results[True], results[False]))
    print("%d nodes, %d edges, %d layers: gradients differ by at most %.2f %% of their norm"
          % (n, graph.n_edges, a.layers, 100 * far))


if __name__ == "__main__":
    main()
