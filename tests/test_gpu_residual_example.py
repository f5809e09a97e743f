"""The residual discriminators of examples/: the gradients of a whole network against 64 bits, training
that learns, and 8-bit scoring near bf16 scoring."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

F64 = torch.float64


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1811_12843_gb300 import _build
    _build.build()
    import residual_discriminators
    return residual_discriminators


def _logits64(p, x, depth):
    def linear(name, v):
        return v @ p[name + ".w"].transpose(-1, -2) + p[name + ".b"][:, None, :]

    def norm(name, v):
        return v * (v.square().mean(dim=-1, keepdim=True) + 1e-6).rsqrt() * p[name][:, None, :]

    s = linear("stem", x)
    for i in range(depth):
        u = linear("%d.up" % i, norm("%d.norm" % i, s))
        s = s + linear("%d.down" % i, torch.nn.functional.gelu(u, approximate="tanh"))
    return linear("head", norm("norm", s))[..., 0]


@pytest.mark.parametrize("cells,rows,x_dim,width,hidden", [(1, 40, 784, 256, 512), (3, 33, 100, 72, 136),
                                                           (2, 17, 50, 31, 45)])
def test_gradients_of_a_network(R, cells, rows, x_dim, width, hidden):
    """bf16 rounds weights, activations and deltas to 2^-8 each; over the eight roundings that lie on a
    path through two blocks the gradients' relative error, in the 2-norm, stays below 8 2^-8."""
    nets = R.ResidualNets(cells, x_dim, width, hidden, depth=2, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((cells, rows, x_dim), generator=gen, device="cuda").to(torch.bfloat16)
    labels = (torch.rand((cells, rows), generator=gen, device="cuda") > 0.5).float()
    logits, saved = nets.forward(x)
    loss, dlogits = R.loss_and_gradient(logits, labels)
    grads = nets.backward(dlogits, saved)
    p = {k: (nets.w[k] if k in nets.w else v).to(F64).requires_grad_(True) for k, v in nets.p.items()}
    ref = _logits64(p, x.to(F64), 2)
    ref_loss = torch.nn.functional.softplus(torch.where(labels > 0, -ref, ref)).mean(dim=1)
    ref_loss.sum().backward()
    assert (logits.to(F64) - ref).norm() < 8 * 2.0 ** -8 * ref.norm()
    assert set(grads) == set(nets.p)
    for k, g in grads.items():
        assert g.shape == nets.p[k].shape and g.dtype == torch.float32
        assert (g.to(F64) - p[k].grad).norm() < 8 * 2.0 ** -8 * p[k].grad.norm(), k


def test_training_learns_and_8_bits_agree(R):
    import lipz_synth
    pool = torch.from_numpy(lipz_synth.blob_pool(5, n=1000, dim=784)).cuda()
    gen = torch.Generator(device="cuda").manual_seed(6)
    nets = R.ResidualNets(4, depth=2)
    opt = R.Adam(nets.p)
    first = None
    for _ in range(25):
        x, labels = R.batch(pool, 4, 64, gen)
        logits, saved = nets.forward(x)
        loss, dlogits = R.loss_and_gradient(logits, labels)
        first = loss if first is None else first
        opt.step(nets.p, nets.backward(dlogits, saved))
        nets.refresh()
    assert (loss < 0.5 * first).all()
    x, labels = R.batch(pool, 4, 64, gen)
    logits = nets.forward(x)[0]
    served = nets.score(x, nets.quantized())
    # 2^-4 of each operand's elements, uncorrelated over the sums: a few percent of the logits
    assert (served - logits).norm() < 0.15 * logits.norm()
    assert ((logits > 0) == (labels > 0)).float().mean() > 0.9
