"""Gradient clipping refuses to write what it reads or writes elsewhere: on
the host, at the C entry (addresses that are never used: every call here is
refused before anything is launched), and from Python on the GPU."""
import ctypes

import pytest
import torch

from paper_2609_28358_amd import mxconv as mx

ARG = -2
F32, BF16 = 0, 1
WS, NORM = 0x100000, 0x200000


def _call(*specs, norm=NORM, ws=WS):
    arr = (ctypes.c_int64 * (4 * len(specs)))(*(v for s in specs for v in s))
    L = mx.lib()
    return L.mxconv_grad_clip(len(specs), arr, 1.0, ctypes.c_void_p(norm), ctypes.c_void_p(ws),
                              L.mxconv_grad_clip_workspace_bytes(), None)


A, B, C, D = 0x1000000, 0x2000000, 0x3000000, 0x4000000


@pytest.mark.parametrize("specs", [
    [(A, B, 8, F32), (B, A, 8, F32)],                         # each into the other
    [(A, A, 8, F32), (A, A, 8, F32)],                         # one twice, in place
    [(A, C, 8, F32), (B, C, 8, F32)],                         # one output for two
    [(A, A, 100, F32), (A + 396, A + 396, 100, F32)],         # slices that share their last and first element
    [(A + 396, A + 396, 100, F32), (A, A, 100, F32)],
    [(A, C, 100, BF16), (B, C + 198, 100, BF16)],
    [(A, A + 4, 8, F32)],                                     # its own source, shifted
    [(A + 4, A, 8, F32)],
    [(A, C, 8, F32), (B, D, 1000, F32), (D + 3996, D + 8000, 1, F32)],        # the last element of a long output is a source
    [(A, C, 8, F32), (B, B, 1000, F32), (B + 400, D, 1, F32)],                # a slice of a tensor that is scaled in place
    [(A + 64 * k, A + 64 * k, 16, F32) for k in range(2000)] + [(A + 640, A + 640, 1, F32)],
    [(A + 64 * (k * 7 % 2000), C + 64 * (k * 7 % 2000), 16, F32) for k in range(2000)] + [(C + 64 * 1999 + 60, D, 1, F32)],
], ids=range(12))
def test_overlaps(specs):
    assert _call(*specs) == ARG


def test_norm_and_workspace():
    assert _call((A, B, 100, F32), norm=A + 4) == ARG
    assert _call((A, B, 100, F32), norm=B + 396) == ARG
    assert _call((A, 0, 100, F32), ws=A - 16) == ARG
    assert _call((A, B, 100, F32), norm=WS + 16) == ARG
    assert _call((A, B, 100, F32), ws=B + 16) == ARG
    assert _call((A, A, 100, F32), ws=A - 16) == ARG


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return "cuda:0"


@pytest.mark.gpu
def test_refused_in_python(gpu):
    a, b, flat = torch.ones(8, device=gpu), torch.full((8,), 2.0, device=gpu), torch.full((1000,), 3.0, device=gpu)
    for call in (lambda: mx.grad_clip([a, b], 1.0, out=[b, a]), lambda: mx.grad_clip([a, a], 1.0),
                 lambda: mx.grad_clip([flat[:500], flat[499:]], 1.0), lambda: mx.grad_clip([flat[:500]], 1.0, out=[flat[1:501]]),
                 lambda: mx.grad_clip([flat[:500], flat[10:20]], 1.0, out=[flat[:500], b.new_empty(10)]),
                 lambda: mx.grad_clip([flat], 1.0, norm_out=flat[7])):
        with pytest.raises(mx.MxconvError):
            call()
    assert (a == 1).all() and (b == 2).all() and (flat == 3).all()


@pytest.mark.gpu
def test_norm_alone_may_lie_in_a_tensor(gpu):
    """Without outputs the norm is written when all has been read."""
    flat = torch.ones(10000, device=gpu)
    assert float(mx.grad_norm([flat], norm_out=flat[77])) == 100.0
    assert flat[77] == 100.0 and int((flat != 1).sum()) == 1


@pytest.mark.gpu
def test_neighbours_are_fine(gpu):
    """Slices that touch, in any order; empty ones anywhere; a source read by
    two; outputs between the sources."""
    flat = torch.arange(1000., device=gpu)
    cuts = [(500, 1000), (0, 499), (499, 500), (250, 250)]
    want = flat / (float(flat.double().norm()) + 1e-6)
    mx.grad_clip([flat[a:b] for a, b in cuts], 1.0)
    assert torch.allclose(flat, want, rtol=1e-6, atol=0)
    buf = torch.ones(400, device=gpu)
    srcs, outs = [buf[0:100], buf[200:300], buf[0:100]], [buf[100:200], buf[300:400], torch.empty(100, device=gpu)]
    norm = float(mx.grad_clip(srcs, 1.0, out=outs))
    assert abs(norm - 300 ** 0.5) < 1e-5
    assert all(torch.allclose(o, torch.full_like(o, 300 ** -0.5), rtol=1e-6, atol=0) for o in outs)
    assert (buf[:100] == 1).all() and (buf[200:300] == 1).all()
