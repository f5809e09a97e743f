"""A population of residual discriminators, trained in bf16 and served in 8 bits.

Every individual tells the rows of a data pool from Gaussian noise with a network deeper than the
grid's own: a stem, `depth` pre-norm residual blocks and a head,

    s = x W0^T + b0
    per block:  h = rmsnorm(s);  s = s + gelu(h W1^T + b1) W2^T + b2
    logit = rmsnorm(s) . w + b

All individuals train at once, each with weights of its own (the operators' groups). Weights are
kept in fp32 with Adam's moments; the products read bf16 copies. Afterwards the weights are quantised
row by row, and the same rows are scored over 8-bit operands.

    python examples/residual_discriminators.py [--cells 12] [--steps 60]
"""

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1811_12843_gb300 import operators as ops

BF16, F32 = torch.bfloat16, torch.float32


class ResidualNets:
    """`cells` networks; parameters are fp32 tensors [cells, ...] by name."""

    def __init__(self, cells, x_dim=784, width=256, hidden=512, depth=3, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.depth, self.p = depth, {}

        def weight(name, n, k):
            self.p[name + ".w"] = torch.randn((cells, n, k), generator=gen, device="cuda") * k ** -0.5
            self.p[name + ".b"] = torch.zeros((cells, n), device="cuda")

        weight("stem", width, x_dim)
        for i in range(depth):
            self.p["%d.norm" % i] = torch.ones((cells, width), device="cuda")
            weight("%d.up" % i, hidden, width)
            weight("%d.down" % i, width, hidden)
        self.p["norm"] = torch.ones((cells, width), device="cuda")
        weight("head", 1, width)
        self.refresh()

    def refresh(self):
        """The bf16 copies that the products read."""
        self.w = {k: v.to(BF16) for k, v in self.p.items() if k.endswith(".w")}

    def forward(self, x):
        """Logits [cells, rows] of x [cells, rows, x_dim], and what the backward pass reads. A block's
        result joins the stream in the norm of the block after it."""
        p, w = self.p, self.w
        delta, stream, kept = ops.linear(x, w["stem.w"], p["stem.b"])[0], None, []
        for i in range(self.depth):
            n = ops.rmsnorm(delta, p["%d.norm" % i], residual=stream, keep=True)
            a, pre = ops.linear(n.y, w["%d.up.w" % i], p["%d.up.b" % i], act="gelu", keep=True)
            delta, stream = ops.linear(a, w["%d.down.w" % i], p["%d.down.b" % i])[0], n.sum
            kept.append((n, a, pre))
        n = ops.rmsnorm(delta, p["norm"], residual=stream, keep=True)
        logits = ops.linear(n.y, w["head.w"], p["head.b"], out_dtype=F32)[0]
        return logits[..., 0], (x, kept, n)

    def backward(self, dlogits, saved):
        """Gradients of every parameter, fp32, from those of the logits."""
        p, w, g = self.p, self.w, {}
        x, kept, n = saved

        def product(name, dy, inp, want_dx=True, **kw):
            dx, g[name + ".w"], g[name + ".b"] = ops.linear_backward(
                dy, inp, w[name + ".w"], want_dx=want_dx, dw_dtype=F32, **kw)
            return dx

        dy = product("head", dlogits[..., None].to(BF16), n.y)
        dstream, g["norm"] = ops.rmsnorm_backward(dy, n.sum, n.rstd, p["norm"])
        for i in reversed(range(self.depth)):
            n, a, pre = kept[i]
            # (dstream reaches both the block's result and the stream beside it)
            da = product("%d.down" % i, dstream, a)
            dh = product("%d.up" % i, da, n.y, act="gelu", pre=pre)
            dstream, g["%d.norm" % i] = ops.rmsnorm_backward(dh, n.sum, n.rstd, p["%d.norm" % i],
                                                             dsum=dstream)
        product("stem", dstream, x, want_dx=False)
        return g

    def quantized(self):
        """The weights in 8 bits with a scale per row."""
        return {k: ops.quantize_rows(v) for k, v in self.w.items()}

    def score(self, x, q):
        """Logits over 8-bit operands; the stream is updated in place."""
        p = self.p

        def product(name, a, **kw):
            return ops.linear(a[0], q[name + ".w"][0], p[name + ".b"], x_scale=a[1],
                              w_scale=q[name + ".w"][1], **kw)[0]

        s = product("stem", ops.quantize_rows(x))
        for i in range(self.depth):
            n = ops.rmsnorm(s, p["%d.norm" % i], e4m3=True)
            a = product("%d.up" % i, (n.y, n.scale), act="gelu")
            product("%d.down" % i, ops.quantize_rows(a), residual=s, out=s)
        n = ops.rmsnorm(s, p["norm"], e4m3=True)
        return product("head", (n.y, n.scale), out_dtype=F32)[..., 0]


class Adam:
    def __init__(self, params, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8):
        self.lr, self.b1, self.b2, self.eps, self.t = lr, beta1, beta2, eps, 0
        self.m = {k: torch.zeros_like(v) for k, v in params.items()}
        self.v = {k: torch.zeros_like(v) for k, v in params.items()}

    def step(self, params, grads):
        self.t += 1
        for k, p in params.items():
            m, v, g = self.m[k], self.v[k], grads[k]
            m.lerp_(g, 1 - self.b1)
            v.mul_(self.b2).addcmul_(g, g, value=1 - self.b2)
            den = (v / (1 - self.b2 ** self.t)).sqrt_().add_(self.eps)
            p.addcdiv_(m, den, value=-self.lr / (1 - self.b1 ** self.t))


def loss_and_gradient(logits, labels):
    """Mean binary cross entropy per individual, and its gradient by the logits."""
    loss = torch.nn.functional.softplus(torch.where(labels > 0, -logits, logits)).mean(dim=1)
    return loss, (torch.sigmoid(logits) - labels) / logits.shape[1]


def batch(pool, cells, rows, gen):
    """Per individual `rows` rows of the pool and as many of noise, and their labels."""
    pick = torch.randint(0, pool.shape[0], (cells, rows), generator=gen, device="cuda")
    noise = 0.5 * torch.randn((cells, rows, pool.shape[1]), generator=gen, device="cuda")
    labels = torch.cat([torch.ones(cells, rows), torch.zeros(cells, rows)], dim=1).cuda()
    return torch.cat([pool[pick], noise], dim=1).to(BF16), labels


def main():
    import lipz_synth
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--cells", type=int, default=12)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rows", type=int, default=100)
    a = ap.parse_args()
    pool = torch.from_numpy(lipz_synth.blob_pool(1811, n=4000, dim=784)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(7)
    nets = ResidualNets(a.cells)
    opt = Adam(nets.p)
    for step in range(a.steps):
        x, labels = batch(pool, a.cells, a.rows, gen)
        logits, saved = nets.forward(x)
        loss, dlogits = loss_and_gradient(logits, labels)
        opt.step(nets.p, nets.backward(dlogits, saved))
        nets.refresh()
        if step % 10 == 0 or step == a.steps - 1:
            print("step %3d  loss %.4f (worst individual %.4f)" % (step, loss.mean(), loss.max()))
    x, labels = batch(pool, a.cells, a.rows, gen)
    logits, q = nets.forward(x)[0], nets.quantized()
    served = nets.score(x, q)
    right = ((logits > 0) == (labels > 0)).float().mean()
    agree = ((logits > 0) == (served > 0)).float().mean()
    print("held-out rows: %.1f %% right in bf16; 8 bits agree on %.1f %%, logits off by %.3f of their rms"
          % (100 * right, 100 * agree, (served - logits).square().mean().sqrt() /
             logits.square().mean().sqrt()))


if __name__ == "__main__":
    main()
