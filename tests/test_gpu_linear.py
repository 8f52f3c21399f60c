"""The linear products on MX matrices against fp64: forward with bias,
activation, residual and the kept pre-activation, both gradients, at sizes
from one row to several tiles, odd sizes, strided outputs, split contractions,
every format pair, padded rows, non-finite blocks, streams and graph replay.
Bounds: mx_matrix.py."""
import numpy as np
import pytest
import torch

import mx_matrix as mm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


def _rand(shape, seed, dtype, std=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def _np(t):
    return t.cpu().to(torch.float64).numpy()


def _fwd_ref(x, w, bias, fn, res):
    z = x @ w.T
    tz = mm.product_tol(x, w)
    if bias is not None:
        z = z + _np(bias)
        tz = tz + mm.U * (np.abs(z) + tz)
    y = mm.act(z, fn)
    ty = 1.1 * tz + (np.abs(y) * (4 + np.abs(z)) * 2.0 ** -23 if fn == 2 else 0)
    if res is not None:
        y = y + _np(res)
        ty = ty + mm.U * (np.abs(y) + ty)
    return z, tz, y, ty


# rows, ins, outs: one row; a few rows; 33..64 rows;
# one 32-block; odd everything; several tiles; a wide tile grid with a ragged edge
SIZES = [(1, 64, 96), (1, 1000, 37), (5, 4500, 70), (31, 32, 33), (47, 260, 300), (64, 2080, 129), (65, 96, 65),
         (130, 1, 1), (200, 777, 515), (700, 333, 1030), (1300, 130, 1250),
         (2100, 200, 1990), (1900, 2030, 260),
         # long contractions of each product, split over workgroups
         (3, 17000, 70), (9000, 40, 70), (40, 70, 17000), (100, 8300, 90)]


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(mx, fmt, size):
    rows, ins, outs = size
    fw, fx = mm.FORMATS[fmt]
    k = SIZES.index(size)
    x, xv = mm.matrix(mx, rows, ins, fx, 10 + k)
    w, wv = mm.matrix(mx, outs, ins, fw, 40 + k, std=ins ** -0.5)
    dtype = (torch.bfloat16, torch.float32)[k % 2]
    bias = _rand((outs,), 70 + k, torch.float32) if k % 3 else None
    res = _rand((rows, outs), 80 + k, dtype) if k % 2 else None
    fn = k % 3
    pre = torch.full((rows, outs), 7.0, dtype=dtype, device=DEV)
    y = mx.linear(w, x, bias=bias, fn=fn, residual=res, dtype=dtype, pre_out=pre)
    z, tz, yr, ty = _fwd_ref(xv, wv, bias, fn, res)
    mm.check(pre, z, tz, dtype, "pre")
    mm.check(y, yr, ty, dtype, "y")
    # without what is optional: the same bits
    y2 = mx.linear(w, x, bias=bias, fn=fn, residual=res, dtype=dtype)
    assert torch.equal(y, y2)


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(mx, fmt, size):
    rows, ins, outs = size
    fg, fx = mm.FORMATS[fmt]
    k = SIZES.index(size)
    x, xv = mm.matrix(mx, rows, ins, fx, 110 + k)
    w, wv = mm.matrix(mx, outs, ins, fg, 140 + k, std=ins ** -0.5)
    dz, gv = mm.matrix(mx, rows, outs, fg, 170 + k, std=1e-3)
    dtype = (torch.bfloat16, torch.float32)[(k + 1) % 2]
    fn = (k + 1) % 3
    z = _rand((rows, ins), 180 + k, dtype, 2.0) if fn else None
    add = _rand((rows, ins), 190 + k, dtype, 1e-3) if k % 2 else None
    dx = mx.linear_dgrad(w, dz, fn=fn, z=z, add=add, dtype=dtype)
    ref, tol = gv @ wv, mm.product_tol(gv, wv.T)
    if fn:
        zz = _np(z)
        d = mm.act_grad(zz, fn)
        # s and z (1 - s) cancel near SiLU's minimum: absolute, (4 + |z|) 2^-22
        tol = tol * (np.abs(d) + 1e-6) + np.abs(ref) * ((4 + np.abs(zz)) * 2.0 ** -22 if fn == 2 else 0)
        ref = ref * d
        tol = tol + mm.U * np.abs(ref)
    if add is not None:
        ref = ref + _np(add)
        tol = tol + mm.U * (np.abs(ref) + tol)
    mm.check(dx, ref, tol, dtype, "dx")
    dw, db = mx.linear_wgrad(dz, x)
    mm.check(dw, gv.T @ xv, mm.product_tol(gv.T, xv.T), torch.float32, "dw")
    mm.check(db, gv.sum(0), (rows / 16 + 32) * 2.0 ** -23 * np.abs(gv).sum(0), torch.float32, "db")
    dw2, none = mx.linear_wgrad(dz, x, bias=False)
    assert none is None and torch.equal(dw, dw2)


def test_gradient_against_differences(mx):
    """dL/dX, dL/dW and dL/db of L = <silu(X W^T + b), C> from the dgrad and
    wgrad calls, against central differences of L in fp64, with values every
    format holds exactly (so quantization changes nothing)."""
    rows, ins, outs = 6, 40, 50
    g = np.random.default_rng(3)
    xv, wv = g.integers(-2, 3, (rows, ins)) * 1.0, g.integers(-2, 3, (outs, ins)) * 0.5
    dzv = g.integers(-2, 3, (rows, outs)) * 1.0
    q = {n: mx.quantize_matrix(torch.tensor(v, dtype=torch.float32, device=DEV), 0)
         for n, v in (("x", xv), ("w", wv), ("dz", dzv))}
    for n, v in (("x", xv), ("w", wv), ("dz", dzv)):
        assert np.array_equal(mm.values(q[n]), v)
    u = g.normal(size=(rows, ins))                   # pre-activation of this layer's X, were X = silu(u)
    dx = mx.linear_dgrad(q["w"], q["dz"], fn=2, z=torch.tensor(u, dtype=torch.float32, device=DEV), dtype=torch.float32)
    u32 = u.astype(np.float32).astype(np.float64)
    dw, db = mx.linear_wgrad(q["dz"], q["x"])
    h = 1e-4

    def loss(u_, w_, b_, x_=None):
        return float((((mm.act(u_, 2) if x_ is None else x_) @ w_.T + b_) * dzv).sum())

    b = np.zeros(outs)
    for i, j in ((0, 0), (3, 17), (5, 39)):
        e = np.zeros_like(u32)
        e[i, j] = h
        d = (loss(u32 + e, wv, b) - loss(u32 - e, wv, b)) / (2 * h)
        assert abs(float(dx[i, j]) - d) <= 1e-5 * max(1.0, abs(d))
    for i, j in ((0, 0), (20, 9), (49, 39)):
        e = np.zeros_like(wv)
        e[i, j] = h
        d = (loss(None, wv + e, b, xv) - loss(None, wv - e, b, xv)) / (2 * h)
        assert abs(float(dw[i, j]) - d) <= 1e-5 * max(1.0, abs(d))
    e = np.zeros(outs)
    e[7] = h
    d = (loss(None, wv, e, xv) - loss(None, wv, -e, xv)) / (2 * h)
    assert abs(float(db[7]) - d) <= 1e-5 * max(1.0, abs(d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_results_larger_than_the_caches(mx, dtype):
    """Whole-line rows of a result past 32 MB are stored past the caches; the
    same product with rows that begin elsewhere gives the same values."""
    rows, ins, outs = 8200, 64, 2048
    x, xv = mm.matrix(mx, rows, ins, 1, 5)
    w, wv = mm.matrix(mx, outs, ins, 1, 6)
    res = _rand((rows, outs), 7, dtype)
    pre = torch.empty((rows, outs), dtype=dtype, device=DEV)
    y = mx.linear(w, x, fn=2, residual=res, dtype=dtype, pre_out=pre)
    z, tz, yr, ty = _fwd_ref(xv, wv, None, 2, res)
    mm.check(pre, z, tz, dtype, "pre")
    mm.check(y, yr, ty, dtype, "y")
    wide = torch.full((rows, outs + 8), 9.0, dtype=dtype, device=DEV)
    mx.linear(w, x, fn=2, residual=res, dtype=dtype, out=wide[:, :outs])
    assert torch.equal(wide[:, :outs], y) and (wide[:, outs:] == 9).all()
    dz, gv = mm.matrix(mx, rows, 64, 1, 8)
    w2, w2v = mm.matrix(mx, 64, outs, 1, 9)
    dx = mx.linear_dgrad(w2, dz, fn=1, z=pre, dtype=dtype)
    ref, tol = gv @ w2v, mm.product_tol(gv, w2v.T)
    on = _np(pre) > 0
    mm.check(dx, ref * on, tol * on, dtype, "dx")


def test_calls_from_two_threads(mx):
    """Concurrent calls on streams of their own equal the sequential ones."""
    import threading
    x, _ = mm.matrix(mx, 9000, 200, 1, 1)
    dz, _ = mm.matrix(mx, 9000, 96, 1, 2)
    w, _ = mm.matrix(mx, 96, 200, 1, 3)
    want = (mx.linear(w, x), *mx.linear_wgrad(dz, x))
    torch.cuda.synchronize()
    got, streams = [None, None], [torch.cuda.Stream() for _ in range(2)]

    def work(k):
        for _ in range(10):
            got[k] = (mx.linear(w, x, stream=streams[k]), *mx.linear_wgrad(dz, x, stream=streams[k]))
        streams[k].synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pad", [1, 4, 13])
def test_strided_rows_and_untouched_columns(mx, dtype, pad):
    """Outputs, residual and pre-activation as column ranges of wider buffers:
    the values of the dense call, and nothing behind a row written."""
    rows, ins, outs = 70, 100, 84
    x, _ = mm.matrix(mx, rows, ins, 1, 5)
    w, _ = mm.matrix(mx, outs, ins, 1, 6)
    res = _rand((rows, outs), 7, dtype)
    pre = torch.empty((rows, outs), dtype=dtype, device=DEV)
    y = mx.linear(w, x, fn=2, residual=res, dtype=dtype, pre_out=pre)
    wide = torch.full((3, rows + 2, outs + pad), 9.0, dtype=dtype, device=DEV)
    wide[2, :rows, :outs] = res
    mx.linear(w, x, fn=2, residual=wide[2, :rows, :outs], dtype=dtype, out=wide[0, :rows, :outs],
              pre_out=wide[1, :rows, :outs]) if (wide[1].data_ptr() | wide[2].data_ptr()) % 16 == 0 else pytest.skip(
                  "rows of this padding leave the buffers unaligned")
    assert torch.equal(wide[0, :rows, :outs], y) and torch.equal(wide[1, :rows, :outs], pre)
    assert (wide[:2, rows:] == 9).all() and (wide[:2, :, outs:] == 9).all()
    # in place on the residual
    mx.linear(w, x, fn=2, residual=wide[2, :rows, :outs], dtype=dtype, out=wide[2, :rows, :outs])
    assert torch.equal(wide[2, :rows, :outs], y)


def test_act_role_matrix_is_the_same_operand(mx):
    m = _rand((64, 100), 3, torch.float32)
    a = mx.quantize(m.view(64, 1, 1, 100), mx.ACT, 1, mx.NHWC)
    b = mx.quantize_matrix(m, 1)
    assert a.shape == b.shape and torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    w, _ = mm.matrix(mx, 50, 100, 1, 4)
    assert torch.equal(mx.linear(w, a), mx.linear(w, b))


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
def test_nonfinite_blocks_stay_where_they_are(mx, fmt):
    """A NaN or infinity makes its 32 x 32 block NaN, and with it exactly the
    outputs that read the block: the 32 rows (a row operand), or the 32
    columns (a weight); zeros elsewhere in the contraction's padding do not
    hide or spread it."""
    fw, fx = mm.FORMATS[fmt]
    rows, ins, outs = 100, 70, 90
    xf, wf = _rand((rows, ins), 1, torch.float32), _rand((outs, ins), 2, torch.float32)
    base = mx.linear(mx.quantize_matrix(wf, fw), mx.quantize_matrix(xf, fx), dtype=torch.float32)
    xf[40, 69] = float("nan")
    wf[10, 0] = float("inf")
    y = mx.linear(mx.quantize_matrix(wf, fw), mx.quantize_matrix(xf, fx), dtype=torch.float32)
    bad = torch.zeros((rows, outs), dtype=torch.bool, device=DEV)
    bad[32:64] = True
    bad[:, :32] = True
    assert torch.equal(torch.isnan(y), bad)
    assert torch.equal(y[~bad], base[~bad])


def test_rows_do_not_see_each_other(mx):
    """A row's results are those of the row computed with other rows, bit for
    bit, whatever the rest of its block holds (same scales)."""
    x = _rand((32, 512), 1, torch.float32)
    w, _ = mm.matrix(mx, 200, 512, 0, 2)
    x[0, :] = x.abs().amax()                       # every block's scale is set by row 0
    y = mx.linear(w, mx.quantize_matrix(x, 0), dtype=torch.float32)
    x2 = x.clone()
    x2[5:] = 0
    y2 = mx.linear(w, mx.quantize_matrix(x2, 0), dtype=torch.float32)
    assert torch.equal(y[:5], y2[:5]) and (y2[5:] == 0).all()


def test_repeated_calls_are_bit_equal(mx):
    """Split contractions are joined in a fixed order."""
    x, _ = mm.matrix(mx, 9000, 200, 0, 1)
    dz, _ = mm.matrix(mx, 9000, 96, 0, 2)
    assert mx.linear_workspace_bytes(mx.LINEAR_WGRAD, 9000, 96, 200) > 0
    first = mx.linear_wgrad(dz, x)
    for _ in range(4):
        again = mx.linear_wgrad(dz, x)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_stream_and_graph(mx):
    """A call on another stream, and a captured forward + backward replayed
    with eager work between the replays, give the eager results."""
    rows, ins, outs = 300, 1100, 260
    x, _ = mm.matrix(mx, rows, ins, 1, 1)
    w, _ = mm.matrix(mx, outs, ins, 1, 2)
    dz, _ = mm.matrix(mx, rows, outs, 1, 3)
    z = _rand((rows, ins), 4, torch.bfloat16)

    def step():
        return (mx.linear(w, x, fn=2), mx.linear_dgrad(w, dz, fn=2, z=z), *mx.linear_wgrad(dz, x))

    want = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = mx.linear(w, x, fn=2, stream=s)
    s.synchronize()
    assert torch.equal(got, want[0])
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k
        step()


def _at(t, k, fill=9.0):
    """(buffer, its view of t's shape k elements in)"""
    buf = torch.full((t.numel() + 16,), fill, dtype=t.dtype, device=t.device)
    v = buf[k:k + t.numel()].view(t.shape)
    return buf, v


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(3, 96, 70), (130, 96, 200), (3, 17000, 70)], ids=lambda s: "x".join(map(str, s)))
def test_pointers_at_any_element(mx, dtype, size):
    """Full-precision operands that begin at odd elements: the bits of aligned
    ones, and nothing written around them."""
    rows, ins, outs = size
    x, _ = mm.matrix(mx, rows, ins, 0, 1)
    w, _ = mm.matrix(mx, outs, ins, 0, 2, std=ins ** -0.5)
    dz, _ = mm.matrix(mx, rows, outs, 0, 3)
    bias, res = _rand((outs,), 4, torch.float32), _rand((rows, outs), 5, dtype)
    z, add = _rand((rows, ins), 6, dtype), _rand((rows, ins), 7, dtype)
    pre = torch.empty_like(res)
    y = mx.linear(w, x, bias=bias, fn=2, residual=res, dtype=dtype, pre_out=pre)
    dx = mx.linear_dgrad(w, dz, fn=2, z=z, add=add, dtype=dtype)
    dw, db = mx.linear_wgrad(dz, x)

    def put(t, k):
        buf, v = _at(t, k)
        v.copy_(t)
        return v

    for k in (1, 3):
        bufs = [_at(t, k) for t in (y, pre, dx, dw, db)]
        o = [v for _, v in bufs]
        mx.linear(w, x, bias=put(bias, k), fn=2, residual=put(res, k + 1), dtype=dtype, out=o[0], pre_out=o[1])
        mx.linear_dgrad(w, dz, fn=2, z=put(z, k + 4), add=put(add, k), dtype=dtype, out=o[2])
        mx.linear_wgrad(dz, x, out=o[3], bias_out=o[4])
        for name, ref, (buf, v) in zip(("y", "pre", "dx", "dw", "db"), (y, pre, dx, dw, db), bufs):
            assert torch.equal(v, ref), name
            assert (buf[:k] == 9).all() and (buf[k + ref.numel():] == 9).all(), name


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1", "e2m3"])
@pytest.mark.parametrize("size", [(333, 700, 2500), (333, 700, 1000), (1300, 600, 1900), (1, 32, 33), (95, 5000, 2112),
                                  (4129, 40, 70), (8200, 40, 33)], ids=lambda s: "x".join(map(str, s)))
def test_column_sums(mx, fmt, size):
    """db by one, two and four workgroups a column block, an odd number of row
    blocks, rows that end inside a block; dw does not depend on it.  Bound as in
    test_backward."""
    rows, ins, outs = size
    f = mm.FORMATS[fmt][0]
    x, _ = mm.matrix(mx, rows, ins, f, 500)
    dz, gv = mm.matrix(mx, rows, outs, f, 501, std=1e-3)
    dw, db = mx.linear_wgrad(dz, x)
    mm.check(db, gv.sum(0), (rows / 16 + 32) * 2.0 ** -23 * np.abs(gv).sum(0), torch.float32, "db")
    assert torch.equal(dw, mx.linear_wgrad(dz, x, bias=False)[0])
    for _ in range(3):
        assert torch.equal(db, mx.linear_wgrad(dz, x)[1])


@pytest.mark.parametrize("fmt", list(mm.FORMATS))
def test_long_contractions_of_small_grids(mx, fmt):
    """One 64 x 64 tile a CU at most, from 40 blocks of the contraction on, in
    every product; ragged in all three sizes, with everything the epilogue takes."""
    fw, fx = mm.FORMATS[fmt]
    for rows, ins, outs in ((100, 1281, 130), (70, 1250, 333), (129, 3001, 65)):
        x, xv = mm.matrix(mx, rows, ins, fx, 510)
        w, wv = mm.matrix(mx, outs, ins, fw, 511, std=ins ** -0.5)
        bias, res = _rand((outs,), 512, torch.float32), _rand((rows, outs), 513, torch.bfloat16)
        pre = torch.empty_like(res)
        y = mx.linear(w, x, bias=bias, fn=2, residual=res, dtype=torch.bfloat16, pre_out=pre)
        z, tz, yr, ty = _fwd_ref(xv, wv, bias, 2, res)
        mm.check(pre, z, tz, torch.bfloat16, "pre")
        mm.check(y, yr, ty, torch.bfloat16, "y")
        # the same sizes with the roles of the products exchanged
        x, xv = mm.matrix(mx, ins, rows, fx, 514)
        dz, gv = mm.matrix(mx, ins, outs, fw, 515, std=1e-3)
        dw, db = mx.linear_wgrad(dz, x)
        mm.check(dw, gv.T @ xv, mm.product_tol(gv.T, xv.T), torch.float32, "dw")
        mm.check(db, gv.sum(0), (ins / 16 + 32) * 2.0 ** -23 * np.abs(gv).sum(0), torch.float32, "db")
        dz, gv = mm.matrix(mx, rows, ins, fw, 516, std=1e-3)
        w, wv = mm.matrix(mx, ins, outs, fw, 517)
        add = _rand((rows, outs), 518, torch.float32, 1e-3)
        dx = mx.linear_dgrad(w, dz, add=add, dtype=torch.float32)
        ref = gv @ wv + _np(add)
        mm.check(dx, ref, mm.product_tol(gv, wv.T) + mm.U * np.abs(ref), torch.float32, "dx")


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1", "e2m3"])
@pytest.mark.parametrize("rows", [70, 97, 321])
def test_nonfinite_column_sums(mx, fmt, rows):
    """A NaN in the last row makes the sums of its block's 32 columns NaN and no
    others: row blocks that do not exist count as zeros."""
    f = mm.FORMATS[fmt][0]
    g = _rand((rows, 100), 1, torch.float32)
    x, _ = mm.matrix(mx, rows, 40, f, 2)
    base = mx.linear_wgrad(mx.quantize_matrix(g, f), x)[1]
    g[rows - 1, 70] = float("nan")
    db = mx.linear_wgrad(mx.quantize_matrix(g, f), x)[1]
    bad = torch.zeros(100, dtype=torch.bool, device=DEV)
    bad[64:96] = True
    assert torch.equal(torch.isnan(db), bad) and torch.equal(db[~bad], base[~bad])
