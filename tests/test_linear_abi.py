"""Linear layers, residual norms and gradient clipping on the host (no GPU):
sizes, and every refusal of the C entry points and of the Python calls.  Calls
here either fail validation or are pure size queries; none reaches a kernel."""
import ctypes

import pytest
import torch

from paper_2609_28358_amd import mxconv as mx

P = ctypes.c_void_p
GOOD = P(0x10000)        # 16-byte aligned, never dereferenced: validation fails first
ODD = P(0x10001)
NULL, ARG, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4, -6


def _lin(rows=64, outs=96, ins=64):
    return ctypes.byref(mx.MxcLinear(rows, outs, ins))


def test_workspace_sizes():
    L = mx.lib()
    for op in (0, 1, 2):
        assert L.mxconv_linear_workspace_bytes(op, _lin()) == 0              # short contractions are not split
    assert L.mxconv_linear_workspace_bytes(2, _lin(9000, 40, 70)) % (40 * 96 * 4) == 0
    assert L.mxconv_linear_workspace_bytes(2, _lin(9000, 40, 70)) > 0
    assert L.mxconv_linear_workspace_bytes(0, _lin(3, 70, 17000)) > 0
    assert L.mxconv_linear_workspace_bytes(1, _lin(3, 17000, 70)) > 0
    assert L.mxconv_linear_workspace_bytes(3, _lin(3, 17000, 70)) == 0
    assert L.mxconv_linear_workspace_bytes(0, _lin(0, 70, 9000)) == 0
    assert L.mxconv_linear_workspace_bytes(0, None) == 0
    assert L.mxconv_grad_clip_workspace_bytes() > 0
    assert mx.norm_workspace_bytes(1, 100) == 0                              # a single workgroup
    full = mx.norm_workspace_bytes(5000, 100)
    assert full > 0
    for kw in (dict(gate=False), dict(post=False), dict(pre=False), dict(gate=False, post=False)):
        assert mx.norm_workspace_bytes(5000, 100, **kw) <= full
    # the workspace does not grow with the rows without bound
    assert mx.norm_workspace_bytes(10 ** 9, 100) == mx.norm_workspace_bytes(10 ** 6, 100)


def _fwd(lin=None, fmt=0, wc=GOOD, ws=GOOD, xc=GOOD, xs=GOOD, bias=None, fn=0, res=None, ldr=0, y=GOOD, ldy=96, z=None, ldz=0,
         dtype=0, wsp=None, wsb=0):
    return mx.lib().mxconv_linear_fwd(lin or _lin(), fmt, wc, ws, xc, xs, bias, fn, res, ldr, y, ldy, z, ldz, dtype, wsp, wsb,
                                      None)


def test_linear_fwd_refusals():
    for name in ("wc", "ws", "xc", "xs", "y"):
        assert _fwd(**{name: None}) == NULL, name
        assert _fwd(**{name: ODD}) == ALIGN, name
    assert mx.lib().mxconv_linear_fwd(None, 0, GOOD, GOOD, GOOD, GOOD, None, 0, None, 0, GOOD, 96, None, 0, 0, None, 0,
                                      None) == NULL
    for fmt in (-1, 4, 3, mx.pair(0, 1), mx.pair(3, 1), 0x20):               # unknown, E3M2 alone, pairs not built
        assert _fwd(fmt=fmt) == ARG, fmt
    assert _fwd(fmt=mx.pair(1, 3), y=ODD) == ALIGN                           # the pair that is built gets past that
    for lin in (_lin(0), _lin(-1), _lin(64, 0), _lin(64, 96, 0)):
        assert _fwd(lin) == ARG
    big = mx.MxcLinear(1, (1 << 20) + 1, 64)
    assert _fwd(ctypes.byref(big), ldy=(1 << 20) + 1) == SHAPE
    assert _fwd(_lin(2 ** 31 - 1, 96, 1 << 20)) == SHAPE                     # more blocks than 32 bits count
    for fn in (3, -1, mx.FN_SILU | mx.FN_PRE_OUT, mx.FN_SILU | mx.FN_BF16):
        assert _fwd(fn=fn) == ARG, fn
    assert _fwd(dtype=2) == ARG
    assert _fwd(ldy=95) == ARG
    assert _fwd(res=P(0x20000), ldr=95) == ARG
    assert _fwd(z=P(0x20000), ldz=95) == ARG
    assert _fwd(z=GOOD, ldz=96) == ARG                                       # z and y are one buffer
    assert _fwd(res=GOOD, ldr=100) == ARG                                    # in place needs one stride
    assert _fwd(bias=ODD) == ALIGN and _fwd(res=ODD, ldr=96) == ALIGN and _fwd(z=ODD, ldz=96) == ALIGN
    long = _lin(3, 70, 17000)
    need = mx.lib().mxconv_linear_workspace_bytes(0, long)
    assert _fwd(long) == WORKSPACE and _fwd(long, wsp=GOOD, wsb=need - 1) == WORKSPACE
    assert _fwd(long, wsp=ODD, wsb=need) == ALIGN


def test_elements_alignment_is_enough():
    """What is checked last for each call is the workspace: full-precision
    operands at any element get that far."""
    long, big = _lin(3, 70, 17000), _norm(rows=5000)
    need = mx.lib().mxconv_linear_workspace_bytes(0, long)
    f4, h2 = P(0x10004), P(0x30002)
    for dtype, a, b in ((0, f4, P(0x20008)), (1, h2, P(0x40006))):
        kw = dict(y=a, ldy=96, bias=f4, res=b, ldr=96, z=P(b.value + 0x1000), ldz=96, dtype=dtype)
        assert _fwd(long, wsp=ODD, wsb=need, **kw) == ALIGN
        assert _fwd(long, wsp=GOOD, wsb=need - 1, **kw) == WORKSPACE
    assert _fwd(y=h2, dtype=0) == ALIGN and _fwd(bias=h2, dtype=1) == ALIGN
    assert mx.lib().mxconv_norm_fwd(_norm(gate=h2), GOOD, 48, GOOD, 48, GOOD, 48, P(0x20000), 48, None) == ALIGN
    assert mx.lib().mxconv_norm_fwd(_norm(), h2, 48, GOOD, 48, GOOD, 48, P(0x20000), 48, None) == ALIGN


def test_linear_dgrad_refusals():
    L = mx.lib()

    def f(lin=None, fmt=0, wc=GOOD, ws=GOOD, gc=GOOD, gs=GOOD, fn=0, z=None, ldz=0, res=None, ldr=0, dx=GOOD, ldx=64, dtype=0):
        return L.mxconv_linear_dgrad(lin or _lin(), fmt, wc, ws, gc, gs, fn, z, ldz, res, ldr, dx, ldx, dtype, None, 0, None)

    for name in ("wc", "ws", "gc", "gs", "dx"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: ODD}) == ALIGN, name
    assert f(fmt=7) == ARG and f(fn=9) == ARG and f(dtype=5) == ARG
    assert f(fn=2) == NULL                                                   # an activation without z
    assert f(fn=2, z=P(0x20000), ldz=63) == ARG and f(ldx=63) == ARG and f(res=P(0x20000), ldr=63) == ARG
    assert f(fn=2, z=GOOD, ldz=80) == ARG
    assert f(fn=2, z=ODD, ldz=64) == ALIGN
    assert f(_lin(64, 96, 0)) == ARG


def test_linear_wgrad_refusals():
    L = mx.lib()

    def f(lin=None, fmt=0, gc=GOOD, gs=GOOD, xc=GOOD, xs=GOOD, dw=GOOD, db=None, wsp=None, wsb=0):
        return L.mxconv_linear_wgrad(lin or _lin(), fmt, gc, gs, xc, xs, dw, db, wsp, wsb, None)

    for name in ("gc", "gs", "xc", "xs", "dw"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: ODD}) == ALIGN, name
    assert f(fmt=mx.pair(3, 1)) == ARG and f(db=ODD) == ALIGN and f(_lin(-5)) == ARG
    assert f(_lin(9000, 40, 70)) == WORKSPACE


def test_rows_near_the_integer_limit():
    """Rows whose rounding up to blocks would pass 31 bits are refused by every
    product, also where they are only the contraction."""
    L = mx.lib()
    for rows in ((1 << 30) + 1, 2 ** 31 - 33, 2 ** 31 - 31, 2 ** 31 - 1):
        lin = _lin(rows, 32, 32)
        assert [L.mxconv_linear_workspace_bytes(op, lin) for op in range(3)] == [0, 0, 0]
        assert L.mxconv_linear_fwd(lin, 1, GOOD, GOOD, GOOD, GOOD, None, 0, None, 0, GOOD, 32, None, 0, 0, None, 0, None) == SHAPE
        assert L.mxconv_linear_dgrad(lin, 1, GOOD, GOOD, GOOD, GOOD, 0, None, 0, None, 0, GOOD, 32, 0, None, 0, None) == SHAPE
        assert L.mxconv_linear_wgrad(lin, 1, GOOD, GOOD, GOOD, GOOD, GOOD, None, GOOD, 1 << 40, None) == SHAPE


def _norm(rows=10, gates=2, d=48, dtype=0, eps=1e-6, post=GOOD, gate=GOOD, pre=GOOD):
    return ctypes.byref(mx.MxcNorm(rows, gates, d, dtype, 1.0, eps, post, gate, pre))


def test_norm_refusals():
    L = mx.lib()

    def f(nm=None, x=GOOD, ldx=48, y=GOOD, ldy=48, h=GOOD, ldh=48, u=P(0x20000), ldu=48):
        return L.mxconv_norm_fwd(nm or _norm(), x, ldx, y, ldy, h, ldh, u, ldu, None)

    def b(nm=None, dh=GOOD, lddh=48, du=GOOD, lddu=48, h=GOOD, ldh=48, y=GOOD, ldy=48, dx=P(0x20000), lddx=48, dy=P(0x30000),
          lddy=48, dp=GOOD, dq=GOOD, dg=GOOD, ws=GOOD, wsb=1 << 30):
        return L.mxconv_norm_bwd(nm or _norm(), dh, lddh, du, lddu, h, ldh, y, ldy, dx, lddx, dy, lddy, dp, dq, dg, ws, wsb,
                                 None)

    for call in (f, b):
        assert call(_norm(rows=0)) == ARG and call(_norm(d=0)) == ARG and call(_norm(dtype=2)) == ARG
        for eps in (-1.0, float("nan"), float("inf")):
            assert call(_norm(eps=eps)) == ARG, eps
        assert call(_norm(gates=0)) == ARG and call(_norm(gates=-2)) == ARG
        assert call(_norm(gates=3)) == SHAPE                                 # does not divide the rows
        assert call(_norm(post=ODD)) == ALIGN and call(_norm(gate=ODD)) == ALIGN and call(_norm(pre=ODD)) == ALIGN
        long = _norm(d=8193)
        lds = {n: 9000 for n in call.__code__.co_varnames if n.startswith("ld")}
        assert call(long, **lds) == SHAPE
    for name in ("x", "y", "h", "u"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: ODD}) == ALIGN, name
    for name in ("ldx", "ldy", "ldh", "ldu"):
        assert f(**{name: 47}) == ARG, name
    assert f(u=GOOD) == ARG and f(ldx=64) == ARG                             # u over h; h in place of x at another stride
    for name in ("dh", "du", "h", "y", "dx", "dy", "dp", "dq", "dg"):
        assert b(**{name: None}) == NULL, name
        assert b(**{name: ODD}) == ALIGN, name
    for name in ("lddh", "lddu", "ldh", "ldy", "lddx", "lddy"):
        assert b(**{name: 47}) == ARG, name
    assert b(dy=P(0x20000)) == ARG and b(dx=GOOD, lddx=64) == ARG and b(dy=GOOD, lddy=64) == ARG
    big = _norm(rows=5000)
    assert b(big, ws=None) == WORKSPACE and b(big, wsb=16) == WORKSPACE and b(big, ws=ODD) == ALIGN


def _tensors(*specs):
    arr = (ctypes.c_int64 * (4 * max(1, len(specs))))()
    for k, (src, dst, n, dt) in enumerate(specs):
        arr[4 * k], arr[4 * k + 1], arr[4 * k + 2], arr[4 * k + 3] = src, dst, n, dt
    return arr


def test_clip_refusals():
    L = mx.lib()
    need = L.mxconv_grad_clip_workspace_bytes()
    ok = (0x10000, 0x20000, 8, 0)

    def f(*specs, count=None, max_norm=1.0, norm=GOOD, ws=GOOD, wsb=need, tensors=True):
        return L.mxconv_grad_clip(len(specs) if count is None else count, _tensors(*specs) if tensors else None, max_norm, norm,
                                  ws, wsb, None)

    assert f(ok, count=-1) == ARG and f(ok, count=65537) == ARG
    for m in (-1.0, float("nan")):
        assert f(ok, max_norm=m) == ARG
    assert f(ok, tensors=False) == NULL and f(ok, ws=None) == NULL and f(ok, wsb=need - 1) == WORKSPACE
    assert f(ok, ws=ODD) == ALIGN and f(ok, norm=P(0x10002)) == ALIGN
    assert f((0, 0x20000, 8, 0)) == NULL and f((0x10002, 0x20000, 8, 0)) == ALIGN and f((0x10000, 0x20001, 8, 1)) == ALIGN
    assert f((0x10002, 0x20004, 8, 1), ws=ODD) == ALIGN                      # bf16 at any element is fine, the workspace is not
    assert f(*[(0x10000 + k, 0, 1 << 36, 0) for k in range(0, 80, 4)]) == SHAPE
    assert f((0x10000, 0x20000, -1, 0)) == ARG and f((0x10000, 0x20000, 8, 2)) == ARG
    assert f(ok, (0x30000, 0, 8, 0)) == ARG                                  # outputs for some tensors only
    assert f((0x10000, 0, 8, 0), norm=None) == NULL                          # nothing to write
    assert L.mxconv_grad_clip(0, None, 1.0, None, GOOD, need, None) == 0     # nothing to do


def _q(rows, cols, fmt=0, role=mx.WEIGHT):
    return mx.MxTensor(torch.zeros(max(1, mx.codes_bytes(mx.WEIGHT, fmt, rows, cols, 1, 1)), dtype=torch.uint8),
                       torch.zeros(max(1, mx.scales_bytes(mx.WEIGHT, fmt, rows, cols, 1, 1)), dtype=torch.uint8), role, fmt,
                       (rows, cols, 1, 1))


def test_python_refusals():
    """Each raises MxconvError before the library is called (CPU tensors would
    be refused last)."""
    E = mx.MxconvError
    w, x, dz = _q(96, 64), _q(40, 64), _q(40, 96)
    cases = [lambda: mx.linear(w, _q(40, 65)), lambda: mx.linear_dgrad(w, _q(40, 95)), lambda: mx.linear_wgrad(dz, _q(41, 64)),
             lambda: mx.linear(_q(40, 64, role=mx.ACT), x), lambda: mx.linear(w, x, bias=torch.zeros(95)),
             lambda: mx.linear(w, x, bias=torch.zeros(96, dtype=torch.float64)),
             lambda: mx.linear(w, x), lambda: mx.linear_dgrad(w, dz), lambda: mx.linear_wgrad(dz, x),      # not on a GPU
             lambda: mx.quantize_matrix(torch.zeros(3, 4, 5), 0),
             lambda: mx.norm_residual(torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.float16)),
             lambda: mx.norm_residual(torch.zeros(4, 8), torch.zeros(4, 8)),
             lambda: mx.norm_residual(torch.zeros(4, 8), torch.zeros(4, 8), gate=torch.zeros(3, 8)),
             lambda: mx.norm_residual(torch.zeros(4, 8), torch.zeros(4, 8), gate=torch.zeros(0, 8)),
             lambda: mx.norm_residual(torch.zeros(4, 8), torch.zeros(4, 8), w_post=torch.zeros(7)),
             lambda: mx.norm_residual_backward(torch.zeros(4, 8), None, None, torch.zeros(4, 8), w_pre=torch.zeros(8)),
             lambda: mx.grad_clip([], 1.0), lambda: mx.grad_clip([torch.zeros(3)], 1.0)]
    short = _q(96, 64)
    short.codes = short.codes[:-1]
    cases.append(lambda: mx.linear(short, x))
    conv = mx.MxTensor(w.codes, w.scales, mx.WEIGHT, 0, (96, 64, 1, 2))
    cases.append(lambda: mx.linear(conv, x))
    for k, c in enumerate(cases):
        with pytest.raises(E):
            c()
            pytest.fail(f"case {k} was not refused")
    # strides, types and sizes of full-precision arguments
    dev = torch.device("cpu")
    t = torch.zeros(4, 16)
    assert mx._rows_cols(t, "t", (4, 16), torch.float32, dev) == 16
    assert mx._rows_cols(t[:, :7], "t", (4, 7), torch.float32, dev) == 16
    assert mx._rows_cols(t[:1, 3:9], "t", (1, 6), torch.float32, dev) == 6
    assert mx._rows_cols(torch.zeros(4, 1).expand(4, 1), "t", (4, 1), torch.float32, dev) == 1
    for bad, shape in ((t[:, ::2], (4, 8)), (t.t(), (16, 4)), (t, (4, 15)), (t.half(), (4, 16))):
        with pytest.raises(E):
            mx._rows_cols(bad, "t", shape, torch.float32, dev)
