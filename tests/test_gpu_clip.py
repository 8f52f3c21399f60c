"""The norm of many tensors and their scaling, against fp64: sizes around the
16-byte vectors and the chunk, empty tensors, more tensors than one launch
takes, mixed types, huge and tiny values, no scaling needed, non-finite
gradients, in place and out of place, graph replay.

The norm is rounded once from fp64 (2^-24 relative, and the sum's own error is
below 2^-40); the factor is rounded to fp32 and the product once more, for
bf16 to bf16."""
import math

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


def _make(sizes, dtypes, std, seed=1):
    g = torch.Generator()
    g.manual_seed(seed)
    return [(torch.randn(n, generator=g) * std).to(dtypes[k % len(dtypes)]).to(DEV) for k, n in enumerate(sizes)]


def _check(mx, ts, max_norm):
    ref = [t.cpu().to(torch.float64).numpy() for t in ts]
    norm = math.sqrt(sum(float((r * r).sum()) for r in ref))
    factor = min(1.0, max_norm / (norm + 1e-6))
    outs = [torch.full_like(t, 3.0) for t in ts]
    got = mx.grad_clip(ts, max_norm, out=outs)
    assert abs(float(got) - norm) <= 2 * mm.U * norm
    for r, o in zip(ref, outs):
        mm.check(o, r * factor, 3 * mm.U * np.abs(r * factor), o.dtype)
    assert float(mx.grad_norm(ts)) == float(got)
    again = [t.clone() for t in ts]
    assert float(mx.grad_clip(again, max_norm)) == float(got)
    assert all(torch.equal(a, o) for a, o in zip(again, outs))
    return norm, outs


F, B = torch.float32, torch.bfloat16
CASES = {"one": ([1], [F]), "odd": ([1, 2, 3, 5, 7, 8, 9, 15, 17, 31], [F, B]),
         "chunk": ([4095, 4096, 4097, 8191, 8192, 8193, 16385], [F, B]), "empty": ([0, 5, 0, 0, 70000, 0], [B, F]),
         "many": ([37 * k % 5000 for k in range(1000)], [F, B, B]), "large": ([3000001, 17, 5000000], [B, F]),
         "long": ([90000001, 33, 20000000], [B, F])}


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("max_norm", [0.5, 1e9, 0.0])
def test_clip(mx, name, max_norm):
    sizes, dt = CASES[name]
    norm, outs = _check(mx, _make(sizes, dt, 1.0), max_norm)
    if max_norm > norm:
        for t, o in zip(_make(sizes, dt, 1.0), outs):
            assert torch.equal(t, o)               # a factor of one copies


@pytest.mark.parametrize("std", [1e30, 1e-30], ids=["huge", "tiny"])
def test_squares_past_fp32(mx, std):
    """Squares that overflow or vanish in fp32: the norm is right, and so is
    the factor."""
    _check(mx, _make([1000, 3000], [F, B], std), 2.0)


def test_all_empty_and_none(mx):
    t = [torch.empty(0, device=DEV), torch.empty((3, 0), device=DEV)]
    assert float(mx.grad_clip(t, 1.0)) == 0.0 and float(mx.grad_norm(t)) == 0.0


def test_nonfinite(mx):
    """An infinity: norm inf, factor 0, its own element NaN (inf * 0), the
    others 0.  A NaN: everything NaN."""
    ts = _make([100, 50], [F, B], 1.0)
    ts[0][3] = float("inf")
    outs = [torch.empty_like(t) for t in ts]
    assert float(mx.grad_clip(ts, 1.0, out=outs)) == float("inf")
    assert torch.isnan(outs[0][3]) and (outs[1] == 0).all() and int(torch.isnan(outs[0]).sum()) == 1
    ts[0][3] = float("nan")
    assert math.isnan(float(mx.grad_clip(ts, 1.0, out=outs)))
    assert torch.isnan(outs[0]).all() and torch.isnan(outs[1]).all()


def test_shapes_views_and_neighbours(mx):
    """Matrices and slices of one buffer; what lies between the slices stays."""
    flat = torch.full((1000,), 2.0, device=DEV)
    a, b = flat[0:333].view(37, 9), flat[400:900]
    norm = float(mx.grad_clip([a, b], 1.0))
    assert abs(norm - 2.0 * math.sqrt(833)) <= 2 * mm.U * norm
    assert (flat[333:400] == 2).all() and (flat[900:] == 2).all() and (flat[:333] < 1).all()


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_any_element_alignment(mx, dtype):
    """Slices that begin at every element offset of a 16-byte vector, with
    lengths around vectors and chunks: the results of aligned copies, and
    the elements between the slices as they were."""
    g = torch.Generator()
    g.manual_seed(3)
    src = torch.randn(60000, generator=g).to(dtype).to(DEV)
    dst = torch.full((60000,), 7.0, dtype=dtype, device=DEV)
    cuts, at = [], 1
    for n in (1, 5, 16, 31, 4096, 4097, 8200, 100, 13, 9001):
        cuts.append((at, n))
        at += n + 2
    ins, outs = [src[a:a + n] for a, n in cuts], [dst[a:a + n] for a, n in cuts]
    assert len({t.data_ptr() % 16 for t in ins}) > 3
    norm = mx.grad_clip(ins, 1.0, out=outs)
    want = [torch.empty_like(t) for t in ins]
    assert float(mx.grad_clip([t.clone() for t in ins], 1.0, out=want)) == float(norm)
    keep = torch.ones(60000, dtype=torch.bool, device=DEV)
    for (a, n), o, w in zip(cuts, outs, want):
        assert torch.equal(o, w)
        keep[a:a + n] = False
    assert (dst[keep] == 7).all()


def test_duplicates_and_mismatches_are_refused(mx):
    a, b = torch.ones(8, device=DEV), torch.ones(8, device=DEV)
    for call in (lambda: mx.grad_clip([a, a], 1.0), lambda: mx.grad_clip([a, b], 1.0, out=[b, b]),
                 lambda: mx.grad_clip([a, b], 1.0, out=[a]), lambda: mx.grad_clip([a], 1.0, out=[torch.ones(7, device=DEV)]),
                 lambda: mx.grad_clip([a, b.bfloat16()], 1.0, out=[a, b]), lambda: mx.grad_clip([a.view(2, 4).t()], 1.0),
                 lambda: mx.grad_clip([a.half()], 1.0), lambda: mx.grad_clip([a, b.cpu()], 1.0),
                 lambda: mx.grad_clip([a], float("nan")), lambda: mx.grad_clip([a], -1.0),
                 lambda: mx.grad_clip([a], 1.0, norm_out=torch.zeros(2, device=DEV)),
                 lambda: mx.grad_clip([a], 1.0, workspace=torch.zeros(8, dtype=torch.uint8, device=DEV))):
        with pytest.raises(mx.MxconvError):
            call()
    assert (a == 1).all() and (b == 1).all()
    # reading one twice is fine: both count
    assert abs(float(mx.grad_norm([a, a])) - 4.0) < 1e-6


def test_graph_replay_reads_new_gradients(mx):
    ts = _make([5000, 7, 130], [F, B], 1.0)
    outs = [torch.empty_like(t) for t in ts]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        mx.grad_clip(ts, 1.0, out=outs)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = mx.grad_clip(ts, 1.0, out=outs)
    for k in range(3):
        for t, n in zip(ts, _make([5000, 7, 130], [F, B], 1.0 + k, seed=k)):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        got, vals = float(norm), [o.clone() for o in outs]
        want = [torch.empty_like(t) for t in ts]
        assert float(mx.grad_clip(ts, 1.0, out=want)) == got
        assert all(torch.equal(a, b) for a, b in zip(vals, want))


def test_norms_kept_in_one_log(mx):
    """norm_out may be any element of a buffer; its neighbours stay."""
    ts = _make([500, 33], [F, B], 1.0)
    log = torch.full((6,), -1.0, device=DEV)
    want = float(mx.grad_norm(ts))
    for k in (1, 3, 4):
        mx.grad_clip(ts, 1e9, norm_out=log[k])
    assert log.tolist() == [-1.0, want, -1.0, want, want, -1.0]


def test_infinite_bound(mx):
    """Never scaled; only with an infinite norm the factor is inf / inf."""
    ts = _make([500, 33], [F, B], 1.0)
    outs = [torch.empty_like(t) for t in ts]
    mx.grad_clip(ts, float("inf"), out=outs)
    assert all(torch.equal(a, b) for a, b in zip(ts, outs))
    ts[1][0] = float("inf")
    assert float(mx.grad_clip(ts, float("inf"), out=outs)) == float("inf")
    assert all(torch.isnan(o).all() for o in outs)
