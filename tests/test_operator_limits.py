"""The largest sizes that the documentation of gradient clipping and of the
linear layers allows, and the first that it does not: on the host, where each
call is refused before a launch, and on the GPU where such tensors fit."""
import ctypes

import pytest
import torch

from paper_2609_28358_amd import mxconv as mx

P = ctypes.c_void_p
ARG, SHAPE, ALIGN, WORKSPACE = -2, -3, -4, -6
WS, NORM, SRC, DST = 0x100000, 0x200000, 1 << 44, 1 << 45
DEV = "cuda:0"


def _clip(*specs):
    arr = (ctypes.c_int64 * (4 * len(specs)))(*(v for s in specs for v in s))
    L = mx.lib()
    return L.mxconv_grad_clip(len(specs), arr, 1.0, P(NORM), P(WS), L.mxconv_grad_clip_workspace_bytes(), None)


def test_clip_sizes():
    """One tensor may have all of the 2^40 elements: the next one's odd address
    is what is refused."""
    odd = (SRC - 2, DST - 8, 1, 0)
    for n in ((1 << 36) + 1, 1 << 37, (1 << 40) - 1):
        assert _clip((SRC, DST, n, 0), odd) == ALIGN, n
        assert _clip((SRC, DST, n, 1), odd) == ALIGN, n
    for n in ((1 << 40) + 1, 1 << 62, (1 << 63) - 1):
        assert _clip((SRC, DST, n, 0)) == SHAPE, n
        assert _clip((SRC, DST, 7, 0), (SRC + 28, DST + 28, n, 0)) == SHAPE, n
    assert _clip((SRC, DST, 1 << 39, 0), (SRC + (1 << 41), DST + (1 << 41), (1 << 39) + 1, 0)) == SHAPE
    assert _clip((SRC, DST, -1, 0)) == ARG


@pytest.mark.gpu
def test_clip_of_more_than_2_36_elements():
    if not torch.cuda.is_available() or torch.cuda.mem_get_info()[0] < 200 << 30:
        pytest.skip("needs 200 GB of device memory")
    n = (1 << 36) + 12345                                                    # 137 GB of bf16, in place
    t = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    marks = [0, (1 << 31) - 1, 1 << 31, 1 << 32, 1 << 35, (1 << 36) - 1, 1 << 36, n - 1]
    for k, i in enumerate(marks):
        t[i] = 3 + k
    norm = float(mx.grad_clip([t], 1.0))
    want = (n + sum((3 + k) ** 2 - 1 for k in range(len(marks)))) ** 0.5
    assert abs(norm - want) <= 2.0 ** -23 * want
    c = torch.tensor(1.0 / (want + 1e-6), dtype=torch.float32)
    for k, i in enumerate(marks):
        assert t[i].item() == ((3 + k) * c).bfloat16().item(), i
    assert t[1].item() == t[n - 2].item() == c.bfloat16().item()
    bad = sum(int((p != t[1]).sum()) for p in t.split(1 << 32))
    assert bad == len(marks)
