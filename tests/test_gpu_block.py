"""The operators of a residual block together (workloads.BlockStep): norm,
quantize, linear with bias and SiLU, quantize, linear with bias and residual,
and back, then the clipping -- each stage's result against fp64 formed from
the stored operands of that stage (the codes it read, the full-precision
tensors it read), so that no bound has to follow an error through a
quantization; the parameter gradients against fp64; the graph replay; and the
clipping at the end of the network steps."""
import numpy as np
import pytest
import torch

import mx_matrix as mm
from paper_2609_28358_amd import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


def _np(t):
    return t.cpu().to(torch.float64).numpy()


def _run(calls):
    for c in calls:
        c[1]()
    torch.cuda.synchronize()


@pytest.mark.parametrize("master", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("fmt", [0, 1, 2], ids=["e4m3", "e2m1", "e2m3"])
@pytest.mark.parametrize("size", [(300, 96, 200), (1, 64, 40), (77, 130, 514)], ids=lambda s: "x".join(map(str, s)))
def test_block_step(mx, fmt, master, size):
    st = wl.BlockStep(*size, fmt, DEV, master=master, clip=None)
    _run(st.calls())
    p = {k: _np(v) for k, v in st.params.items()}
    # quantized operands are those of the tensors they were made from
    for q, t in ((st.w1, st.params["w1"]), (st.u_q, st.u), (st.a_q, st.a), (st.do_q, st.do), (st.dz_q, st.dz)):
        again = mx.quantize_matrix(t, fmt)
        n = mx.codes_bytes(mx.WEIGHT, fmt, *q.shape) - (16 if fmt >= 2 else 0)
        assert torch.equal(again.codes[:n], q.codes[:n]) and torch.equal(again.scales, q.scales)
    w1, w2, u, a, do, dz = (mm.values(t) for t in (st.w1, st.w2, st.u_q, st.a_q, st.do_q, st.dz_q))
    z = u @ w1.T + p["b1"]
    tz = mm.product_tol(u, w1)
    tz = tz + mm.U * (np.abs(z) + tz)
    mm.check(st.z, z, tz, master, "z")
    act = mm.act(z, 2)
    mm.check(st.a, act, 1.1 * tz + np.abs(act) * (4 + np.abs(z)) * 2.0 ** -23, master, "a")
    o = a @ w2.T + p["b2"] + _np(st.h)
    mm.check(st.o, o, mm.product_tol(a, w2) + 3 * mm.U * (np.abs(o) + np.abs(_np(st.h))), master, "o")
    zz = _np(st.z)
    d, r = mm.act_grad(zz, 2), do @ w2
    mm.check(st.dz, r * d, mm.product_tol(do, w2.T) * (np.abs(d) + 1e-6) + np.abs(r) * (5 + np.abs(zz)) * 2.0 ** -22, master,
             "dz")
    mm.check(st.du, dz @ w1, mm.product_tol(dz, w1.T), master, "du")
    rows = size[0]
    for name, g, x in (("2", do, a), ("1", dz, u)):
        mm.check(st.grads["w" + name], g.T @ x, mm.product_tol(g.T, x.T), torch.float32, "dw" + name)
        mm.check(st.grads["b" + name], g.sum(0), (rows / 16 + 32) * 2.0 ** -23 * np.abs(g).sum(0), torch.float32, "db" + name)
    for t in (st.h, st.u, st.dx, st.dy, *st.grads.values()):
        assert torch.isfinite(t).all() and t.abs().max() > 0


def test_block_step_clips_and_replays(mx):
    st = wl.BlockStep(200, 128, 256, 1, DEV, clip=None)
    _run(st.calls())
    plain = {k: v.clone() for k, v in st.grads.items()}
    norm = float(np.sqrt(sum((_np(v) ** 2).sum() for v in plain.values())))
    limit = norm / 3
    st = wl.BlockStep(200, 128, 256, 1, DEV, clip=limit)
    calls = st.calls()
    _run(calls)
    assert abs(float(st.clip.norm) - norm) <= 2 * mm.U * norm
    factor = limit / (norm + 1e-6)
    for k, v in plain.items():
        mm.check(st.grads[k], _np(v) * factor, 4 * mm.U * np.abs(_np(v)) * factor, torch.float32, k)
    want = [t.clone() for t in (st.o, st.dx, st.dy, *st.grads.values())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(calls)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in calls:
            c[1]()
    for k in range(3):
        out = (st.o, st.dx, st.dy, *st.grads.values())
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), k
        _run(calls)


def test_network_steps_clip(mx):
    """The clipping at the end of the network and replay steps: the gradients
    of the step without it, scaled; everything before it unchanged."""
    for make in (lambda clip: wl.NetStep(wl.yolo_net(64), 32, mx.E2M1, DEV, clip=clip),
                 lambda clip: wl.QlrStep(DEV, buffer=64, batch=64, clip=clip)):
        a = make(None)
        ca = a.calls()
        assert ca[-1][0].startswith("wgrad_reduce")
        _run(ca)
        gw = list(a.gw.values()) if isinstance(a.gw, dict) else a.gw
        norm = float(np.sqrt(sum((_np(g) ** 2).sum() for g in gw)))
        b = make(norm / 2)
        _run(b.calls())
        gb = list(b.gw.values()) if isinstance(b.gw, dict) else b.gw
        assert abs(float(b.clip.norm) - norm) <= 2 * mm.U * norm
        factor = (norm / 2) / (norm + 1e-6)
        for x, y in zip(gw, gb):
            mm.check(y, _np(x) * factor, 4 * mm.U * np.abs(_np(x)) * factor, torch.float32)
