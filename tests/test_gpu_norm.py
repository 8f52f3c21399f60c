"""The residual norms against fp64, forward and backward: row lengths around
every thread shape, odd lengths, gates by channel and by group, absent
weights, strides, in-place outputs, zero rows, and graph replay.

Bounds.  A sum of d squares held by 16 values a thread, wave and workgroup
sums: at most 16 + 6 + 8 roundings, so r(v) is off by less than (16 + 4) 2^-24
relative (half of it through the square root, 4 for the division and root),
taken as C = 32.  N(v) multiplies twice more.  U is normalized from an H that
is off absolutely, so its bound scales H's.  The mean of t . hh may cancel: it
is bounded by the mean of magnitudes."""
import numpy as np
import pytest
import torch

import mx_matrix as mm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = 32 * mm.U
EPS = 1e-6


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


def _rand(shape, seed, dtype, std=1.0, mean=0.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(dtype).to(DEV)


def _np(t):
    return None if t is None else t.cpu().to(torch.float64).numpy()


def _rs(v):
    return 1 / np.sqrt((v * v).mean(1, keepdims=True) + EPS)


# rows, d, gates (0: none), post, pre
CASES = [(1, 1, 0, True, True), (1, 1000, 1, True, True), (3, 16, 3, True, True), (7, 64, 1, True, False),
         (50, 255, 5, True, True), (33, 1024, 1, False, True), (12, 1025, 4, True, True), (9, 1032, 0, True, True),
         (40, 4096, 2, True, True), (5, 4097, 1, True, True), (6, 8192, 3, True, True), (4, 8191, 0, False, True),
         (2100, 40, 1, True, True), (3000, 24, 1500, True, True), (1024, 128, 1024, True, True), (10, 48, 2, False, False)]


def _case(case, dtype, seed):
    rows, d, gates, post, pre = case
    x, y = _rand((rows, d), seed, dtype), _rand((rows, d), seed + 1, dtype, 2.0)
    wp = _rand((d,), seed + 2, torch.float32, 0.2, 1.0) if post else None
    wq = _rand((d,), seed + 3, torch.float32, 0.2, 1.0) if pre else None
    g = _rand((gates, d), seed + 4, torch.float32) if gates else None
    return x, y, wp, wq, g


def _gate(g, rows):
    return 1.0 if g is None else np.repeat(_np(g), rows // g.shape[0], axis=0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}g{c[2]}{'p' if c[3] else ''}{'q' if c[4] else ''}")
def test_forward(mx, dtype, case):
    x, y, wp, wq, g = _case(case, dtype, 100 * CASES.index(case))
    h, u = mx.norm_residual(x, y, w_post=wp, gate=g, scale=0.7, w_pre=wq, eps=EPS)
    X, Y = _np(x), _np(y)
    n = Y * _rs(Y) * _np(wp) if wp is not None else Y
    s = float(np.float32(0.7))
    b = s * _gate(g, case[0]) * n
    H = X + b
    tol = C * np.abs(b) + mm.U * np.abs(H)
    mm.check(h, H, tol, dtype, "h")
    if wq is None:
        assert u is None
        return
    r = _rs(H)
    # H's error moves U directly and through r(H), by at most its own mean relative size
    shift = np.sqrt((tol * tol).mean(1, keepdims=True)) * r
    mm.check(u, H * r * _np(wq), (tol * r + np.abs(H) * r * (C + shift)) * np.abs(_np(wq)), dtype, "u")


def _bwd_ref(dh, du, h, y, wp, wq, g, s):
    rows, d = y.shape
    out = {}
    dx, tx = dh.copy(), np.zeros_like(dh)
    if wq is not None:
        r = _rs(h)
        hh, t = h * r, du * wq
        m, ma = (t * hh).mean(1, keepdims=True), np.abs(t * hh).mean(1, keepdims=True)
        dx = dh + r * (t - hh * m)
        tx = mm.U * np.abs(dx) + r * (C * np.abs(t) + np.abs(hh) * 3 * C * ma)
        out["dw_pre"] = ((du * hh).sum(0), 3 * C * np.abs(du * hh).sum(0))
    gg = 1.0 if g is None else np.repeat(g, rows // g.shape[0], axis=0)
    b, tb = s * gg * dx, np.abs(s * gg) * (tx + 2 * mm.U * np.abs(dx))
    ry = _rs(y) if wp is not None else 1.0
    yh = y * ry
    p = yh * wp if wp is not None else y
    if wp is not None:
        q = b * wp
        tq = tb * np.abs(wp) + mm.U * np.abs(q)
        m = (q * yh).mean(1, keepdims=True)
        tm = ((tq + C * np.abs(q)) * np.abs(yh)).mean(1, keepdims=True) * 2
        out["dw_post"] = ((b * yh).sum(0), ((tb + 3 * C * np.abs(b)) * np.abs(yh)).sum(0))
        dy = ry * (q - yh * m)
        ty = ry * (tq + C * np.abs(q) + np.abs(yh) * (tm + 3 * C * np.abs(m)))
    else:
        dy, ty = b, tb
    if g is not None:
        k = (s * dx * p).reshape(g.shape[0], -1, d)
        tk = (np.abs(s) * (tx + 3 * C * np.abs(dx)) * np.abs(p)).reshape(g.shape[0], -1, d)
        out["dgate"] = (k.sum(1), tk.sum(1))
    out["dx"], out["dy"] = (dx, tx), (dy, ty)
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}g{c[2]}{'p' if c[3] else ''}{'q' if c[4] else ''}")
def test_backward(mx, dtype, case):
    """The column sums' bound adds one rounding a row that a thread takes (at
    most 3000 / 256 + 1), one for each of a workgroup's up to 8 rows at a time,
    512 / 32 in a thread of the join and 32 over its threads: 69, within the
    160 below."""
    rows, d = case[:2]
    seed = 100 * CASES.index(case) + 50
    h, y, wp, wq, g = _case(case, dtype, seed)
    dh, du = _rand((rows, d), seed + 5, dtype, 1e-3), _rand((rows, d), seed + 6, dtype, 1e-3)
    got = dict(zip(("dx", "dy", "dw_pre", "dw_post", "dgate"),
                   mx.norm_residual_backward(dh, du if wq is not None else None, h if wq is not None else None, y, w_post=wp,
                                             gate=g, scale=0.7, w_pre=wq, eps=EPS)))
    ref = _bwd_ref(_np(dh), _np(du), _np(h), _np(y), _np(wp), _np(wq), _np(g), float(np.float32(0.7)))
    for name, t in got.items():
        if name not in ref:
            assert t is None, name
            continue
        r, tol = ref[name]
        if name.startswith("dw") or name == "dgate":
            tol = tol * 2 + 160 * mm.U * np.abs(tol) / (3 * C)      # tol / 3C bounds the sum of magnitudes
        mm.check(t, r, tol, torch.float32 if t.dtype == torch.float32 else dtype, name)


def test_gradient_against_differences(mx):
    rows, d = 4, 24
    g = np.random.default_rng(5)
    t = {n: g.normal(size=(rows, d)) for n in ("x", "y", "ch", "cu")}
    w = {n: 1 + 0.2 * g.normal(size=d) for n in ("post", "pre")}
    gate = g.normal(size=(2, d))
    f32 = lambda a: torch.tensor(a, dtype=torch.float32, device=DEV)    # noqa: E731
    for k in (t, w):
        for n in k:
            k[n] = k[n].astype(np.float32).astype(np.float64)
    gate = gate.astype(np.float32).astype(np.float64)

    def forward(x, y, post, pre, gt):
        H = x + 0.5 * np.repeat(gt, 2, axis=0) * (y * _rs(y) * post)
        return H, H * _rs(H) * pre

    def loss(**ch):
        a = dict(x=t["x"], y=t["y"], post=w["post"], pre=w["pre"], gt=gate)
        a.update(ch)
        H, U = forward(**a)
        return float((H * t["ch"] + U * t["cu"]).sum())

    H, _ = forward(t["x"], t["y"], w["post"], w["pre"], gate)
    dx, dy, dq, dp, dg = mx.norm_residual_backward(f32(t["ch"]), f32(t["cu"]), f32(H), f32(t["y"]), w_post=f32(w["post"]),
                                                   gate=f32(gate), scale=0.5, w_pre=f32(w["pre"]), eps=EPS)
    e = 1e-5
    for name, base, got in (("x", t["x"], dx), ("y", t["y"], dy), ("post", w["post"], dp), ("pre", w["pre"], dq),
                            ("gt", gate, dg)):
        for k in (0, base.size // 2, base.size - 1):
            p, m = base.copy().reshape(-1), base.copy().reshape(-1)
            p[k] += e
            m[k] -= e
            diff = (loss(**{name: p.reshape(base.shape)}) - loss(**{name: m.reshape(base.shape)})) / (2 * e)
            assert abs(float(got.reshape(-1)[k]) - diff) <= 2e-5 * max(1.0, abs(diff)), (name, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pad", [8, 3])
def test_strides_in_place_and_untouched_columns(mx, dtype, pad):
    rows, d = 21, 1104
    x, y, wp, wq, g = _case((rows, d, 1, True, True), dtype, 9)
    h, u = mx.norm_residual(x, y, w_post=wp, gate=g, w_pre=wq)
    buf = torch.full((rows, 4 * (d + pad)), 5.0, dtype=dtype, device=DEV)
    v = [buf[:, k * (d + pad):k * (d + pad) + d] for k in range(4)]
    if any(t.data_ptr() % 16 for t in v):
        v = [torch.full((rows, d + pad), 5.0, dtype=dtype, device=DEV)[:, :d] for _ in range(4)]
    v[0].copy_(x)
    v[1].copy_(y)
    mx.norm_residual(v[0], v[1], w_post=wp, gate=g, w_pre=wq, h_out=v[2], u_out=v[3])
    # the scalar path adds in another order than the vectors: within a step of each other
    for a, b in ((v[2], h), (v[3], u)):
        assert torch.allclose(a.float(), b.float(), rtol=2 * torch.finfo(dtype).eps, atol=1e-6)
    mx.norm_residual(v[0], v[1], w_post=wp, gate=g, w_pre=wq, h_out=v[0], u_out=v[3])
    assert torch.equal(v[0], v[2])
    if buf.data_ptr() == v[0].data_ptr():
        assert all((buf[:, k * (d + pad) + d:(k + 1) * (d + pad)] == 5).all() for k in range(4))
    dh, du = _rand((rows, d), 1, dtype), _rand((rows, d), 2, dtype)
    want = mx.norm_residual_backward(dh, du, h, y, w_post=wp, gate=g, w_pre=wq)
    a, b = dh.clone(), y.clone()
    got = mx.norm_residual_backward(a, du, h, b, w_post=wp, gate=g, w_pre=wq, dx_out=a, dy_out=b)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and got[0] is a and got[1] is b


def test_zero_rows_and_nan_rows(mx):
    """A row of zeros gives zeros (r is eps^-1/2); a NaN stays in its row."""
    x, y, wp, wq, g = _case((8, 300, 1, True, True), torch.float32, 3)
    x[2] = 0
    y[2] = 0
    y[5, 7] = float("nan")
    h, u = mx.norm_residual(x, y, w_post=wp, gate=g, w_pre=wq)
    assert (h[2] == 0).all() and (u[2] == 0).all() and torch.isnan(u[5]).all()
    ok = torch.ones(8, dtype=torch.bool)
    ok[5] = False
    assert torch.isfinite(h[ok]).all() and torch.isfinite(u[ok]).all()


def test_graph_replay(mx):
    x, y, wp, wq, g = _case((700, 512, 2, True, True), torch.bfloat16, 3)
    dh, du = _rand((700, 512), 1, torch.bfloat16), _rand((700, 512), 2, torch.bfloat16)

    def step():
        h, u = mx.norm_residual(x, y, w_post=wp, gate=g, w_pre=wq)
        return (h, u, *mx.norm_residual_backward(dh, du, h, y, w_post=wp, gate=g, w_pre=wq))

    want = [t.clone() for t in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [37, 1030])
def test_pointers_at_any_element(mx, dtype, d):
    """Operands, parameters and results that begin at odd elements: the bits of
    aligned ones, and nothing written around them."""
    rows = 24
    case = (rows, d, 3, True, True)
    x, y, wp, wq, g = _case(case, dtype, 900)
    dh, du = _rand((rows, d), 910, dtype), _rand((rows, d), 911, dtype)
    kw = dict(scale=0.7, eps=EPS)
    h, u = mx.norm_residual(x, y, w_post=wp, gate=g, w_pre=wq, **kw)
    grads = mx.norm_residual_backward(dh, du, h, y, w_post=wp, gate=g, w_pre=wq, **kw)

    def at(t, k):
        buf = torch.full((t.numel() + 16,), 9.0, dtype=t.dtype, device=DEV)
        return buf, buf[k:k + t.numel()].view(t.shape)

    def put(t, k):
        v = at(t, k)[1]
        v.copy_(t)
        return v

    def same(ref, bufs, k):
        for t, (buf, v) in zip(ref, bufs):
            assert torch.equal(t, v)
            assert (buf[:k] == 9).all() and (buf[k + t.numel():] == 9).all()

    for k in (1, 3):
        p = dict(w_post=put(wp, k), gate=put(g, k + 1), w_pre=put(wq, k + 2), **kw)
        outs = [at(t, k) for t in (h, u)]
        mx.norm_residual(put(x, k), put(y, k + 1), h_out=outs[0][1], u_out=outs[1][1], **p)
        same((h, u), outs, k)
        bufs = [at(t, k) for t in grads]
        o = [v for _, v in bufs]
        mx.norm_residual_backward(put(dh, k), put(du, k + 1), put(h, k + 2), put(y, k), dx_out=o[0], dy_out=o[1],
                                  dw_pre_out=o[2], dw_post_out=o[3], dgate_out=o[4], **p)
        same(grads, bufs, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(1100, 2048), (1100, 2112), (4200, 520)])
def test_results_of_several_mebibytes(mx, dtype, rows, d):
    """Results in whole cache lines (and rows of 520, which are none in bf16):
    the bits of the same results at one element past a line, and of strided
    ones, whose padding stays."""
    case = (rows, d, 2, True, True)
    x, y, wp, wq, g = _case(case, dtype, 950)
    dh, du = _rand((rows, d), 960, dtype), _rand((rows, d), 961, dtype)
    kw = dict(w_post=wp, gate=g, w_pre=wq, scale=0.7, eps=EPS)
    h, u = mx.norm_residual(x, y, **kw)
    dx, dy = mx.norm_residual_backward(dh, du, h, y, **kw)[:2]
    off = [torch.empty(rows * d + 1, dtype=dtype, device=DEV)[1:].view(rows, d) for _ in range(4)]
    wide = [torch.full((rows, d + 128), 9.0, dtype=dtype, device=DEV) for _ in range(4)]
    for o in (off, [w[:, :d] for w in wide]):
        mx.norm_residual(x, y, h_out=o[0], u_out=o[1], **kw)
        mx.norm_residual_backward(dh, du, h, y, dx_out=o[2], dy_out=o[3], **kw)
        for a, b in zip((h, u, dx, dy), o):
            assert torch.equal(a, b)
    for w in wide:
        assert (w[:, d:] == 9).all()
    ref = _bwd_ref(*(_np(t[:8]) for t in (dh, du, h, y)), _np(wp), _np(wq), _np(g[:1]), float(np.float32(0.7)))
    mm.check(dx[:8], *ref["dx"], dtype, "dx")
    mm.check(dy[:8], *ref["dy"], dtype, "dy")
