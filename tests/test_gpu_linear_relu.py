"""The linear layers' ReLU and its gradient on values that are not finite: a
NaN stays one, as SiLU's does, and where the pre-activation is not positive
the gradient is zero whatever the product is.  On one tile, on tiles whose
waves share the contraction, and on split contractions."""
import pytest
import torch

import mx_matrix as mm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [(100, 70, 90), (20, 200, 90), (3, 17000, 70), (300, 1400, 200)]


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


def _normal(shape, seed, dtype=torch.float32):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(mx, size, fmt, dtype):
    rows, ins, outs = size
    fw, fx = mm.FORMATS[fmt]
    x, w, bias, res = _normal((rows, ins), 1), _normal((outs, ins), 2), _normal((outs,), 3), _normal((rows, outs), 4, dtype)
    bias[7] = float("nan")
    w[40, ins - 1] = float("inf")                    # its block's rows: columns 32 .. 63
    w, x = mx.quantize_matrix(w, fw), mx.quantize_matrix(x, fx)
    z = torch.empty((rows, outs), dtype=dtype, device=DEV)
    y = mx.linear(w, x, bias=bias, fn=mx.FN_RELU, residual=res, dtype=dtype, pre_out=z)
    bad = torch.zeros((rows, outs), dtype=torch.bool, device=DEV)
    bad[:, 7] = True
    bad[:, 32:64] = True
    assert torch.equal(torch.isnan(z), bad) and torch.equal(torch.isnan(y), bad)
    on = (z > 0) & ~bad                              # elsewhere the activation is a zero
    assert torch.equal(y[~on & ~bad], res[~on & ~bad]) and on.any()
    bare = mx.linear(w, x, bias=bias, fn=mx.FN_RELU, dtype=dtype)
    assert torch.equal(bare[on], z[on]) and (bare[~on & ~bad] == 0).all() and torch.isnan(bare[bad]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_input_gradient(mx, size, fmt, dtype):
    rows, outs, ins = size
    fw, fg = mm.FORMATS[fmt]
    w, dz, z, add = _normal((outs, ins), 1), _normal((rows, outs), 2), _normal((rows, ins), 3, dtype), _normal((rows, ins), 4, dtype)
    w[5, 40] = float("nan")                          # its block's columns: 32 .. 63
    w, dz = mx.quantize_matrix(w, fw), mx.quantize_matrix(dz, fg)
    z[0, :] = 0
    z[1, 3:50] = float("nan")
    z[2, 3:50] = float("-inf")
    z[2, 50:] = float("inf")
    v = mx.linear_dgrad(w, dz, dtype=dtype)
    bad = torch.zeros((rows, ins), dtype=torch.bool, device=DEV)
    bad[:, 32:64] = True
    assert torch.equal(torch.isnan(v), bad)
    dx = mx.linear_dgrad(w, dz, fn=mx.FN_RELU, z=z, dtype=dtype)
    off = z <= 0
    assert (dx[off] == 0).all()
    assert torch.equal(dx[~off & ~bad], v[~off & ~bad]) and torch.isnan(dx[~off & bad]).all()
    dx = mx.linear_dgrad(w, dz, fn=mx.FN_RELU, z=z, add=add, dtype=dtype)
    assert torch.equal(dx[off], add[off]) and torch.equal(torch.isnan(dx), bad & ~off)
