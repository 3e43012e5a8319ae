"""The packed product with an activation and a residual in its epilogue, in every kernel that runs products, against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24                    # half a step of fp32, relative


@pytest.fixture(scope="module")
def amq():
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    from paper_1802_00150_b200 import amq as binding
    return binding


def packed(amq, gen, rows, n, k):
    codes = amq.pack(torch.randn((rows, k, n), device="cuda", generator=gen))
    return codes, torch.rand((rows, k), device="cuda", generator=gen) + 0.1


ACTIVATIONS = {
    "NONE": lambda v: v, "RELU": lambda v: v.clamp(min=0), "GELU": lambda v: 0.5 * v * torch.erfc(-v / math.sqrt(2)),
    "SILU": lambda v: v * torch.sigmoid(v), "TANH": torch.tanh, "SIGMOID": torch.sigmoid,
}


def expected(amq, W, x, n, bias, name, residual):
    """(result, allowed error): the product folds k_w k_a exact integers with two roundings each and as many sums, then the bias; an activation
    passes an error on at most 1.13-fold and is itself within 8 roundings (erfc, exp and tanh of CUDA are within 2 to 4 units; silu and gelu are three
    operations more); the residual adds one.  The tensor-core kernels fold sums over whole steps of 256 positions, the padding included (up to `pad` more than
    D), and take the padding's part off after: the folded numbers are up to |D| + pad, and the part taken off is pad once more."""
    D = amq.binary_dots(W[0], x[0], n).double()                             # (batch, m, k_w, k_a), exact
    terms = W[1].double()[None, :, :, None] * x[1].double()[:, None, None, :] * D
    pad = -n % 256
    y = terms.sum((2, 3))
    size = (W[1].double()[None, :, :, None] * x[1].double()[:, None, None, :] * (D.abs() + 2 * pad)).sum((2, 3))
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    out = ACTIVATIONS[name](y)
    k2 = W[0].shape[1] * x[0].shape[1]
    allowed = 1.13 * (2 * k2 + 2) * EPS * size + 8 * EPS * out.abs() + 1e-37
    if residual is not None:
        out = out + residual.double()
        allowed = allowed + EPS * out.abs()
    return out, allowed


# the matrix-vector kernel (whole and ragged chunks, one and two per lane), CUDA cores, streaming and resident tensor-core kernels
SHAPES = [(1, 1, 1), (33, 100, 1), (1000, 1024, 1), (515, 5000, 1), (70, 9000, 1), (7, 40, 3), (300, 256, 5), (129, 300, 15), (2048, 256, 200),
          (1024, 1024, 64), (650, 650, 20), (4100, 1024, 100), (9999, 650, 33), (2048, 8192, 40), (32768, 256, 2), (129, 127, 1024)]


@pytest.mark.parametrize("m,n,batch", SHAPES)
@pytest.mark.parametrize("name", list(ACTIVATIONS))
def test_against_the_definition(amq, m, n, batch, name):
    gen = torch.Generator(device="cuda").manual_seed(m + n + batch)
    kw, ka = 1 + (m + n) % 4, 1 + (n + batch) % 4
    W, x = packed(amq, gen, m, n, kw), packed(amq, gen, batch, n, ka)
    W = W[0], W[1] / math.sqrt(n)           # (results of about 1: no activation is saturated)
    bias = torch.randn(m, device="cuda", generator=gen)
    residual = torch.randn((batch, m), device="cuda", generator=gen)
    for b, r in ((bias, residual), (None, residual), (bias, None)):
        y = amq.binary_gemm_act(*W, *x, n, bias=b, activation=getattr(amq, "ACT_" + name), residual=r)
        ref, allowed = expected(amq, W, x, n, b, name, r)
        assert ((y.double() - ref).abs() <= allowed).all()


@pytest.mark.parametrize("m,n,batch", SHAPES)
def test_alone_it_is_the_product(amq, m, n, batch):
    gen = torch.Generator(device="cuda").manual_seed(1)
    W, x = packed(amq, gen, m, n, 3), packed(amq, gen, batch, n, 2)
    bias = torch.randn(m, device="cuda", generator=gen)
    assert torch.equal(amq.binary_gemm_act(*W, *x, n, bias=bias), amq.binary_gemm(*W, *x, n, bias=bias))


@pytest.mark.parametrize("m,n,batch", [(1000, 1024, 1), (300, 256, 5), (1024, 1024, 64), (4100, 1024, 100), (2048, 256, 200)])
@pytest.mark.parametrize("offset,spare", [(0, 4), (1, 5), (3, 2)])
def test_strides_and_in_place(amq, m, n, batch, offset, spare):
    """Rows of residual and result at any stride and offset; the residual may be the result; what lies between rows stays."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    W, x = packed(amq, gen, m, n, 2), packed(amq, gen, batch, n, 2)
    wide = torch.randn((batch, offset + m + spare), device="cuda", generator=gen)
    residual = wide[:, offset:offset + m]
    ref, allowed = expected(amq, W, x, n, None, "RELU", residual.contiguous())
    out = torch.full((batch, m + 7), 5.0, device="cuda")
    amq.binary_gemm_act(*W, *x, n, activation=amq.ACT_RELU, residual=residual, y=out[:, 2:2 + m])
    assert ((out[:, 2:2 + m].double() - ref).abs() <= allowed).all()
    assert (out[:, :2] == 5).all() and (out[:, 2 + m:] == 5).all()
    before = wide.clone()
    amq.binary_gemm_act(*W, *x, n, activation=amq.ACT_RELU, residual=residual, y=residual)
    assert ((residual.double() - ref).abs() <= allowed).all()
    assert torch.equal(wide[:, :offset], before[:, :offset]) and torch.equal(wide[:, offset + m:], before[:, offset + m:])


@pytest.mark.parametrize("batch", [1, 3, 64])
def test_values_that_saturate(amq, batch):
    """Results far out on both sides: no NaN from an activation, and the exact limits."""
    n = 64
    W = amq.pack(torch.stack([torch.ones((1, n)), -torch.ones((1, n))]).cuda().float()), torch.full((2, 1), 100.0, device="cuda")
    x = amq.pack(torch.ones((batch, 1, n), device="cuda")), torch.ones((batch, 1), device="cuda")
    for name, hi, lo in (("RELU", 6400.0, 0.0), ("GELU", 6400.0, 0.0), ("SILU", 6400.0, 0.0), ("TANH", 1.0, -1.0), ("SIGMOID", 1.0, 0.0)):
        y = amq.binary_gemm_act(*W, *x, n, activation=getattr(amq, "ACT_" + name))
        assert (y[:, 0] == hi).all() and (y[:, 1] == lo).all(), name


@pytest.mark.parametrize("m,n,batch", [(4, 64, 1), (4, 64, 3), (2048, 256, 200), (1024, 1024, 64)])
def test_infinite_sums(amq, m, n, batch):
    """The activations' limits, and NaN as NaN."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    W, x = packed(amq, gen, m, n, 2), packed(amq, gen, batch, n, 2)
    inf = float("inf")
    bias = torch.tensor([inf, -inf, float("nan"), 3e38], device="cuda").repeat(m // 4)
    for name, hi, lo in (("NONE", inf, -inf), ("RELU", inf, 0.0), ("GELU", inf, 0.0), ("SILU", inf, 0.0), ("TANH", 1.0, -1.0), ("SIGMOID", 1.0, 0.0)):
        y = amq.binary_gemm_act(*W, *x, n, bias=bias, activation=getattr(amq, "ACT_" + name))
        assert (y[:, 0::4] == hi).all() and (y[:, 1::4] == lo).all() and torch.isnan(y[:, 2::4]).all(), name
        assert (y[:, 3::4] == (min(hi, bias[3]))).all(), name


def test_refused_tensors(amq):
    gen = torch.Generator(device="cuda").manual_seed(3)
    W, x = packed(amq, gen, 8, 64, 2), packed(amq, gen, 2, 64, 2)
    for residual in (torch.zeros((2, 7), device="cuda"), torch.zeros((2, 8)), torch.zeros((2, 8), device="cuda", dtype=torch.float64),
                     torch.zeros((8, 2), device="cuda").T):
        with pytest.raises(TypeError):
            amq.binary_gemm_act(*W, *x, 64, residual=residual)
    with pytest.raises(amq.AmqError):
        amq.binary_gemm_act(*W, *x, 64, activation=6)
