"""A rectified feed-forward block with experts, as a language model decodes with it.

    python examples/rectified_ffn.py [--tokens 8] [--width 2048] [--hidden 1408] [--experts 64] [--slots 8]

Each token's hidden state is added to the residual stream and normalised, in 8
bits for the products and in its own type for the router; the router picks its
experts; their first products run on 4-bit weights with the rectifier fused, and
their second products skip the zeros that it left.  Weights are random, packed
once.  The program checks the block against elementary torch operations, runs a
few decoding steps, captures a step in a HIP graph, and takes one step of the
router's and the norm's training.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1704_07724_amd as isc  # noqa: E402

FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


class RectifiedExperts:
    """norm -> router -> experts' first products, rectified -> second products over the nonzeros."""

    def __init__(self, width, hidden, experts, slots, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        self.slots = slots
        self.norm = 1 + 0.1 * draw(width)
        self.router = draw(width, experts) * width ** -0.5
        self.bias = 0.01 * draw(experts)
        self.plain = (isc.isc_w4_quantize(draw(experts, hidden, width) * width ** -0.5),
                      isc.isc_w4_quantize(draw(experts, width, hidden) * hidden ** -0.5))
        self.up = isc.isc_w4_pack_codes(*self.plain[0], layout="tiles")
        self.down = isc.isc_w4_pack_codes(*self.plain[1], layout="rows")

    def __call__(self, x, residual):
        """(block's output, residual stream, hidden activations, route, norm) of x [T, width] bfloat16."""
        n = isc.isc_rmsnorm(x, self.norm, residual=residual, mx8=True, rstd=True)
        # torch's product: isc_gemm_f32's tiles are the convolutions', a hundred times as
        # wide as a router, and take 94 us for one token of 2048 and 64 experts
        logits = n.y.float() @ self.router
        route = isc.isc_route(logits, self.slots, bias=self.bias, score="sigmoid")
        u = isc.isc_w4_linear(n.mx8, self.up, route=route, relu=True)
        return isc.isc_w4_skip(u, self.down, route=route), n.h, u, route, n

    def reference(self, n, route):
        """The experts' part by elementary operations on the values that the codes stand for."""
        table = torch.tensor(FP4, device="cuda")

        def dense(codes, scales):
            v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)
            return v * torch.repeat_interleave(scales.float(), 32, -1)[..., : v.shape[-1]]

        x = n.mx8.q.float() * torch.repeat_interleave(n.mx8.scales.float(), 32, -1)[:, : n.mx8.q.shape[1]]
        y = torch.zeros_like(x)
        for t, ids in enumerate(route.ids.tolist()):
            for e, w in zip(ids, route.weights[t]):
                u = torch.relu(dense(*(v[e] for v in self.plain[0])) @ x[t]).bfloat16().float()
                y[t] += w * (dense(*(v[e] for v in self.plain[1])) @ u)
        return y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 8), ("width", 2048), ("hidden", 1408), ("experts", 64), ("slots", 8), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args(argv)
    block = RectifiedExperts(a.width, a.hidden, a.experts, a.slots)
    x = torch.randn((a.tokens, a.width), device="cuda").bfloat16()
    residual = torch.randn_like(x)

    y, h, u, route, n = block(x, residual)
    want = block.reference(n, route)
    err = float((y.float() - want).norm() / want.norm())
    print("block against elementary operations: relative error %.2g; zeros in the hidden layer: %.2f"
          % (err, float((u == 0).float().mean())))

    # decoding: the output is the next step's x, h its residual
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        block(x, residual)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, state = block(x, residual)[:2]
        x.copy_(out)
        residual.copy_(state)
    for name, step in (("eager", lambda: block(x, residual)), ("graph", graph.replay)):
        step()
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(a.steps):
            step()
        torch.cuda.synchronize()
        print("%s: %.1f us a block of %d tokens" % (name, (time.perf_counter() - t) / a.steps * 1e6, a.tokens))

    # training: a gradient that reaches the routing weights goes on to the router and the norm
    y, h, u, route, n = block(x, residual)
    dweights = torch.randn_like(route.weights)
    dlogits = isc.isc_route_bwd(dweights, n.y.float() @ block.router, route.ids, score="sigmoid")
    drouter = n.y.float().t() @ dlogits
    dy = (dlogits @ block.router.t()).bfloat16()
    dx, dnorm = isc.isc_rmsnorm_bwd(dy, n.h, block.norm, n.rstd)
    print("gradients: router %.3g, norm %.3g, hidden state %.3g"
          % (float(drouter.norm()), float(dnorm.norm()), float(dx.float().norm())))
    return err


if __name__ == "__main__":
    sys.exit(0 if main() < 0.01 else 1)
