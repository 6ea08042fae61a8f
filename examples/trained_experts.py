"""A rectified feed-forward block with experts, trained, and then served on 4-bit weights.

    python examples/trained_experts.py [--tokens 512] [--width 256] [--hidden 384] [--experts 16] [--slots 2] [--steps 20]

Every step routes a batch, runs the experts' first products (rectified) and their
second ones (summed under the routing weights), takes the gradients of both, of the
routing weights and of the router, and moves the experts' matrices by their
gradients with momentum, orthogonalised.  The targets are those of another block of
the same kind.  The program checks the gradients against autograd on the same
values, and at the end runs the trained block on packed 4-bit weights.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1704_07724_amd as isc  # noqa: E402


class Experts:
    """router -> first products, rectified -> second products, summed; and its training step."""

    def __init__(self, width, hidden, experts, slots, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        self.slots = slots
        self.router = draw(width, experts) * width ** -0.5
        self.up = (draw(experts, hidden, width) * width ** -0.5).bfloat16()
        self.down = (draw(experts, width, hidden) * hidden ** -0.5).bfloat16()
        self.momentum = [torch.zeros_like(self.up, dtype=torch.float32), torch.zeros_like(self.down, dtype=torch.float32)]

    def forward(self, x):
        logits = x.float() @ self.router
        route = isc.isc_route(logits, self.slots, score="sigmoid")
        u = isc.isc_expert_linear(x, self.up, route, relu=True)
        return isc.isc_expert_linear(u, self.down, route, combine=True), (x, logits, route, u)

    def backward(self, dout, kept):
        """(dx, the gradients of the first and second matrices, of the router)."""
        x, logits, route, u = kept
        second = isc.isc_expert_linear_bwd(dout, u, self.down, route, combine=True)
        first = isc.isc_expert_linear_bwd(second.dx, x, self.up, route, y=u)
        dlogits = isc.isc_route_bwd(second.dweights, logits, route.ids, score="sigmoid")
        dx = first.dx.float() + dlogits @ self.router.t()
        return dx, first.dw, second.dw, x.float().t() @ dlogits

    def move(self, dup, ddown, drouter, rate):
        for weights, grad, m in zip((self.up, self.down), (dup, ddown), self.momentum):
            m.mul_(0.9).add_(grad)
            size = max(1.0, weights.shape[1] / weights.shape[2]) ** 0.5
            weights.copy_(weights.float() - rate * size * isc.isc_orthogonalize(m).float())
        self.router -= rate * drouter / drouter.norm().clamp_min(1e-12)


def reference(block, x, dout):
    """The gradients by autograd, in 64 bits, on the same weights and the same choice of experts."""
    ids = isc.isc_route(x.float() @ block.router, block.slots, score="sigmoid").ids.long()
    xd, up, down, router = (v.double().requires_grad_(True) for v in (x, block.up, block.down, block.router))
    s = torch.sigmoid(torch.gather(xd @ router, 1, ids))
    u = torch.relu((up[ids] * xd[:, None, None, :]).sum(-1))
    y = ((down[ids] * u[:, :, None, :]).sum(-1) * (s / s.sum(-1, keepdim=True))[..., None]).sum(1)
    y.backward(dout.double())
    return xd.grad, up.grad, down.grad, router.grad


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("tokens", 512), ("width", 256), ("hidden", 384), ("experts", 16), ("slots", 2), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args(argv)
    block = Experts(a.width, a.hidden, a.experts, a.slots, 0)
    target = Experts(a.width, a.hidden, a.experts, a.slots, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    batch = lambda n: torch.randn((n, a.width), generator=g, device="cuda").bfloat16()  # noqa: E731

    x, dout = batch(16), batch(16)
    got = block.backward(dout, block.forward(x)[1])
    errors = [float((p.double() - q).norm() / q.norm()) for p, q in zip(got, reference(block, x, dout))]
    print("gradients against autograd: hidden state %.2g, first matrices %.2g, second %.2g, router %.2g" % tuple(errors))

    for step in range(a.steps):
        x = batch(a.tokens)
        y, kept = block.forward(x)
        off = y.float() - target.forward(x)[0].float()
        if step % 5 == 0 or step == a.steps - 1:
            print("step %d: loss %.4f" % (step, float(off.square().mean())))
        block.move(*block.backward((2.0 / a.width * off).bfloat16(), kept)[1:], rate=0.02)

    x = batch(4)
    y, (_, _, route, _) = block.forward(x)
    up = isc.isc_w4_pack_codes(*isc.isc_w4_quantize(block.up), layout="tiles")
    down = isc.isc_w4_pack_codes(*isc.isc_w4_quantize(block.down), layout="rows")
    served = isc.isc_w4_skip(isc.isc_w4_linear(x, up, route=route, relu=True), down, route=route)
    print("served on 4-bit weights: %.2g of the output's norm off" % float((served.float() - y.float()).norm() / y.float().norm()))
    return max(errors)


if __name__ == "__main__":
    sys.exit(0 if main() < 0.03 else 1)
