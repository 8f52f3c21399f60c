"""The 128 x 128 and the 256 x 128 tile of the linear products, every format
pair and product, over contractions long enough that the copies of a coming
stage are issued between the products of the current one and the ring wraps
several times, with a last stage that is not full and edges that end inside a
32-block.

Operands are small integers times a power of two of their 32 x 32 block, which
every format holds exactly, so every partial sum is an integer below 2^24: the
products are exact in fp32 whatever their order, and results are compared bit
for bit with fp64's."""
import pytest
import torch

import mx_matrix as mm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# output rows x columns (32-blocks 130 x 129: 33 x 17 = 561 tiles of 4 x 8 blocks, at least 512;
# 66 x 65: 9 x 17 = 153 such tiles, but 17 x 17 = 289 of 4 x 4, at least 256)
TILES = {"256x128": (4130, 4100), "128x128": (2100, 2050)}
CON = 1365                                 # 43 blocks: 10 stages of four and one of three, or 21 of two and one of one


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


def _ints(mx, rows, cols, fmt, seed):
    """A matrix of integers up to 12 in magnitude and its MX form."""
    g = torch.Generator()
    g.manual_seed(seed)
    up = [(n + 31) // 32 for n in (rows, cols)]
    v = torch.randint(-3, 4, (rows, cols), generator=g).double()
    s = 2.0 ** torch.randint(0, 3, up, generator=g).double()
    v = v * s.repeat_interleave(32, 0).repeat_interleave(32, 1)[:rows, :cols]
    q = mx.quantize_matrix(v.float().to(DEV), fmt)
    assert (mm.values(q) == v.numpy()).all()
    return q, v.to(DEV)


def _whole(shape, seed, dtype, hi=9):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randint(-hi, hi + 1, shape, generator=g).to(dtype).to(DEV)


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("tile", list(TILES))
def test_forward(mx, tile, fmt):
    rows, outs = TILES[tile]
    fw, fx = mm.FORMATS[fmt]
    (x, xv), (w, wv) = _ints(mx, rows, CON, fx, 1), _ints(mx, outs, CON, fw, 2)
    bias = _whole((outs,), 3, torch.float32)
    z = xv @ wv.t() + bias.double()
    assert z.abs().max() < 2 ** 23
    for dtype, fn in ((torch.float32, 1), (torch.bfloat16, 0)):
        res, pre = _whole((rows, outs), 4, dtype), torch.empty((rows, outs), dtype=dtype, device=DEV)
        y = mx.linear(w, x, bias=bias, fn=fn, residual=res, dtype=dtype, pre_out=pre)
        assert torch.equal(pre, z.to(dtype))
        assert torch.equal(y, ((z.clamp(min=0) if fn else z) + res.double()).to(dtype))
        assert torch.equal(mx.linear(w, x, dtype=dtype), (z - bias.double()).to(dtype))


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("tile", list(TILES))
def test_input_gradient(mx, tile, fmt):
    rows, ins = TILES[tile]
    fw, fg = mm.FORMATS[fmt]
    (g, gv), (w, wv) = _ints(mx, rows, CON, fg, 11), _ints(mx, CON, ins, fw, 12)
    ref = gv @ wv
    for dtype in (torch.float32, torch.bfloat16):
        z, add = _whole((rows, ins), 13, dtype), _whole((rows, ins), 14, dtype)
        dx = mx.linear_dgrad(w, g, fn=1, z=z, add=add, dtype=dtype)
        assert torch.equal(dx, (ref * (z > 0) + add.double()).to(dtype))
        assert torch.equal(mx.linear_dgrad(w, g, dtype=dtype), ref.to(dtype))


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("tile", list(TILES))
def test_weight_gradient(mx, tile, fmt):
    outs, ins = TILES[tile]
    fg, fx = mm.FORMATS[fmt]
    (g, gv), (x, xv) = _ints(mx, CON, outs, fg, 21), _ints(mx, CON, ins, fx, 22)
    dw, db = mx.linear_wgrad(g, x)
    assert torch.equal(dw, (gv.t().contiguous() @ xv).float())
    assert torch.equal(db, gv.sum(0).float())
    assert torch.equal(mx.linear_wgrad(g, x, bias=False)[0], dw)
