"""Activations over their whole range, in every kernel that runs products: coefficients of zero leave the bias as the sum, so the argument is exact."""
import pytest
import torch

from test_gpu_product_act import amq, packed  # noqa: F401

pytestmark = pytest.mark.gpu

BATCHES = [1, 3, 64, 512]           # the matrix-vector kernel, CUDA cores, the streaming and the resident tensor-core kernels


def activated(amq, values, batch, name):
    gen = torch.Generator(device="cuda").manual_seed(batch)
    W, x = packed(amq, gen, len(values), 256, 2), packed(amq, gen, batch, 256, 2)
    y = amq.binary_gemm_act(W[0], torch.zeros_like(W[1]), *x, 256, bias=values, activation=getattr(amq, "ACT_" + name))
    assert torch.equal(y, y[:1].expand_as(y))
    return y[0].double()


@pytest.mark.parametrize("batch", BATCHES)
def test_gelu(amq, batch):  # noqa: F811
    """Relative to the result itself, in both tails: the polynomial is within 1.5e-7; its evaluation, the quotient and the exponential add 3 to 4 units of
    2^-23 each at most, 1e-6 in all; the exponent v^2 / 2 is rounded three times (the square, its product with log2(e), and that constant), each 2^-25 v^2."""
    v = torch.linspace(-12.0, 12.0, 32768, device="cuda")
    got = activated(amq, v, batch, "GELU")
    want = v.double() * 0.5 * torch.special.erfc(v.double() * -0.5 ** 0.5)      # (ndtr is 1 + erf, nothing below 1e-16)
    assert ((got - want).abs() <= (1e-6 + 3 * 2.0 ** -25 * v.double() ** 2) * want.abs()).all()


@pytest.mark.parametrize("batch", BATCHES)
def test_silu_and_sigmoid(amq, batch):  # noqa: F811
    """The exponential and the quotient are within 2 units of 2^-23 each, the sum within half of one, the product within half: 5 2^-23."""
    v = torch.linspace(-80.0, 80.0, 32768, device="cuda")
    for name in ("SILU", "SIGMOID"):
        want = torch.special.expit(v.double()) * (v.double() if name == "SILU" else 1.0)
        assert ((activated(amq, v, batch, name) - want).abs() <= 5 * 2.0 ** -23 * want.abs()).all(), name
