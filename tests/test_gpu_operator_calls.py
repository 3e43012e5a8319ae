"""The Python calls of a decoder step's operators: numbers beyond the C call's types."""
import pytest
import torch

from test_gpu_product_act import amq, packed  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("activation", [-1, 6, 1 << 31, 1 << 32, (1 << 32) + 1, -(1 << 32), 1 << 62])
def test_activations_that_are_none(amq, activation):  # noqa: F811
    """An activation beyond 32 bits is refused as any other unknown one, not cut to one that exists."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    W, x = packed(amq, gen, 8, 64, 2), packed(amq, gen, 2, 64, 2)
    with pytest.raises(amq.AmqError) as refused:
        amq.binary_gemm_act(*W, *x, 64, activation=activation)
    assert refused.value.status == -2
    with pytest.raises(OverflowError):
        amq.binary_gemm_act(*W, *x, 64, activation=1 << 64)
