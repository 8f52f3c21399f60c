"""The residual norms where a thread takes several rows of its run, forward
and backward, every result against fp64: runs that cross the border of two
gates' rows (forward), column sums over several rows and over several whole
gates of a workgroup (backward), one row a gate at every row length's shape,
and rows of odd strides with what lies behind them.

Bounds: test_gpu_norm.py.  The column sums' bound adds one rounding for every
row that a thread takes (ITERATIONS below: at most 8), one for each of a
workgroup's up to 8 rows at a time, 512 / 32 in a thread of the join and 32
over its threads: 64, within the 160 below."""
import numpy as np
import pytest
import torch

import mx_matrix as mm
import test_gpu_norm as tn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


# rows, d, gates (0: none), post, pre: rows of a run and how many of them a thread takes, backward and forward
CASES = [(9000, 64, 1, True, True),        # 18 rows, 8 at a time: 3; 9 rows, 4 at a time: 3
         (9000, 61, 0, True, False),       # the same without a gate and without U
         (9000, 1024, 3, True, True),      # 18 rows, 4 at a time: 5; 5 rows, one at a time
         (16384, 1024, 1, False, True),    # 32 rows, 4 at a time: 8; 8 rows
         (2200, 1030, 2, True, True),      # 5 rows, 2 at a time: 3; 3 rows
         (1100, 2112, 2, True, True),      # 3 rows; 3 rows, the border of the gates (550) inside a run
         (1100, 8192, 1, True, True),      # 5 rows; 3 rows
         (12000, 64, 600, True, True),     # two whole gates of 20 rows, 8 at a time: 6; 12 rows, 4 at a time, gates inside
         (3000, 1027, 750, True, True),    # two whole gates of 4 rows, 2 at a time: 4
         (1400, 2050, 700, False, True),   # two whole gates of 2 rows: 4
         (1400, 4096, 700, True, False)]
# one row a gate: each gate's rows are a workgroup's, or two gates' are
CASES += [(n, d, n, True, True) for n in (300, 700) for d in (64, 513, 1025, 2049, 4096, 4097, 8192)]
IDS = [f"{c[0]}x{c[1]}g{c[2]}{'p' if c[3] else ''}{'q' if c[4] else ''}" for c in CASES]


@DTYPES
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(mx, dtype, case):
    x, y, wp, wq, g = tn._case(case, dtype, 31 * CASES.index(case))
    h, u = mx.norm_residual(x, y, w_post=wp, gate=g, scale=0.7, w_pre=wq, eps=tn.EPS)
    X, Y = tn._np(x), tn._np(y)
    b = float(np.float32(0.7)) * tn._gate(g, case[0]) * (Y * tn._rs(Y) * tn._np(wp) if wp is not None else Y)
    H = X + b
    tol = tn.C * np.abs(b) + mm.U * np.abs(H)
    mm.check(h, H, tol, dtype, "h")
    if wq is None:
        assert u is None
        return
    r = tn._rs(H)
    shift = np.sqrt((tol * tol).mean(1, keepdims=True)) * r
    mm.check(u, H * r * tn._np(wq), (tol * r + np.abs(H) * r * (tn.C + shift)) * np.abs(tn._np(wq)), dtype, "u")


@DTYPES
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_backward(mx, dtype, case):
    rows, d = case[:2]
    seed = 31 * CASES.index(case) + 7
    h, y, wp, wq, g = tn._case(case, dtype, seed)
    dh, du = tn._rand((rows, d), seed + 5, dtype, 1e-3), tn._rand((rows, d), seed + 6, dtype, 1e-3)
    pre = wq is not None
    got = dict(zip(("dx", "dy", "dw_pre", "dw_post", "dgate"),
                   mx.norm_residual_backward(dh, du if pre else None, h if pre else None, y, w_post=wp, gate=g, scale=0.7,
                                             w_pre=wq, eps=tn.EPS)))
    ref = tn._bwd_ref(*(tn._np(t) for t in (dh, du, h, y, wp, wq, g)), float(np.float32(0.7)))
    for name, t in got.items():
        if name not in ref:
            assert t is None, name
            continue
        r, tol = ref[name]
        if name.startswith("dw") or name == "dgate":
            tol = tol * 2 + 160 * mm.U * np.abs(tol) / (3 * tn.C)
        mm.check(t, r, tol, torch.float32 if name.startswith("dw") or name == "dgate" else dtype, name)


@DTYPES
@pytest.mark.parametrize("rows,d,pad", [(21, 1104, 3), (21, 1104, 8), (50, 37, 1), (13, 4099, 5), (1100, 512, 1)])
def test_rows_of_odd_strides(mx, dtype, rows, d, pad):
    """Every operand and result a column range of one buffer, so that rows begin
    at any element: the bits of the dense call, in place too, and nothing
    written between the ranges."""
    case = (rows, d, 1, True, True)
    x, y, wp, wq, g = tn._case(case, dtype, 77)
    dh, du = tn._rand((rows, d), 78, dtype), tn._rand((rows, d), 79, dtype)
    kw = dict(w_post=wp, gate=g, w_pre=wq, scale=0.7, eps=tn.EPS)
    h, u = mx.norm_residual(x, y, **kw)
    want = mx.norm_residual_backward(dh, du, h, y, **kw)
    w = d + pad
    buf = torch.full((rows, 8 * w), 5.0, dtype=dtype, device=DEV)
    v = [buf[:, k * w:k * w + d] for k in range(8)]
    for dst, src in zip(v, (x, y, dh, du)):
        dst.copy_(src)
    mx.norm_residual(v[0], v[1], h_out=v[4], u_out=v[5], **kw)
    assert torch.equal(v[4], h) and torch.equal(v[5], u)
    got = mx.norm_residual_backward(v[2], v[3], v[4], v[1], dx_out=v[6], dy_out=v[7], **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for src, k in ((x, 0), (y, 1), (dh, 2), (du, 3)):
        assert torch.equal(v[k], src)
    mx.norm_residual_backward(v[2], v[3], v[4], v[1], dx_out=v[2], dy_out=v[1], **kw)
    assert torch.equal(v[2], want[0]) and torch.equal(v[1], want[1])
    v[1].copy_(y)
    mx.norm_residual(v[0], v[1], h_out=v[0], u_out=v[5], **kw)
    assert torch.equal(v[0], h) and torch.equal(v[5], u)
    assert all((buf[:, k * w + d:(k + 1) * w] == 5).all() for k in range(8))
