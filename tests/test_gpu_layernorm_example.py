"""The residual discriminators of examples/ with layer norms, keeping what their backward pass reads in bf16 or in 8
bits: the gradients of a whole network against 64 bits, and the commands."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")
sys.path.insert(0, EXAMPLES)

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
        off = v - v.mean(dim=-1, keepdim=True)
        return off * (off.square().mean(dim=-1, keepdim=True) + 1e-5).rsqrt() * p[name][:, None, :] + \
            p[name + ".b"][:, None, :]

    s = linear("stem", x)
    for i in range(depth):
        u = linear("%d.up" % i, norm("%d.norm" % i, s))
        s = s + linear("%d.down" % i, torch.nn.functional.gelu(u, approximate="tanh"))
    return linear("head", norm("norm", s))[..., 0]


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("cells,rows,x_dim,width,hidden", [(1, 40, 784, 256, 512), (3, 33, 100, 72, 136),
                                                           (2, 17, 50, 31, 45)])
def test_gradients_of_a_network(R, cells, rows, x_dim, width, hidden, keep8):
    """bf16 rounds weights, activations and deltas to 2^-8 each: over the eight roundings that lie on a path through two
    blocks the gradients' relative error, in the 2-norm, stays below 8 2^-8. Of what is kept in 8 bits an element is off
    by up to 2^-7 of its block's largest; a path meets five such (two sums, two pre-activations, a norm's result), and
    an rms error of half of that or less in each: five 2^-7 more, times 1.5 where the activations that gelu takes from
    rounded pre-activations meet those pre-activations' slopes."""
    nets = R.ResidualNets(cells, x_dim, width, hidden, depth=2, seed=3, norm="layer", keep8=keep8)
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
    tol = 8 * 2.0 ** -8 + (1.5 * 5 * 2.0 ** -7 if keep8 else 0)
    for k, g in grads.items():
        assert g.shape == nets.p[k].shape and g.dtype == torch.float32
        assert (g.to(F64) - p[k].grad).norm() < tol * p[k].grad.norm(), k


def test_checkpoints_need_the_layer_norm(R):
    with pytest.raises(ValueError):
        R.ResidualNets(1, keep8=True)


@pytest.mark.parametrize("args", [("--norm", "layer"), ("--norm", "layer", "--keep", "int8")])
def test_the_commands_run(R, args):
    r = subprocess.run([sys.executable, os.path.join(EXAMPLES, "residual_discriminators.py"), "--cells", "2", "--steps",
                        "3"] + list(args), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "held-out rows" in r.stdout, r.stderr[-2000:]
