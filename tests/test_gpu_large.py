"""Linear products, residual norms and clipping on tensors past 2^31 elements
(byte offsets past 2^32): rows from both sides of every border equal the same
rows computed alone."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = (1 << 20) + 45                     # times 2080 columns: 2.18e9 elements


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    from paper_2609_28358_amd import mxconv
    mxconv.lib()
    return mxconv


def _blocks():
    """First rows of 32-row blocks: the ends, and around 2^30 and 2^31 elements."""
    last = ROWS // 32 * 32 - 32
    return sorted({0, last} | {min(b // 2080 // 32 * 32 + k, last) for b in (1 << 30, 1 << 31) for k in (0, 32)})


def test_linear_outputs_past_32_bits(mx):
    """fp4 values of small integers: every product and sum is exact, so the
    tile shape does not matter to the bits."""
    ins, outs = 64, 2080
    g = torch.Generator(DEV).manual_seed(1)
    x = torch.randint(-3, 4, (ROWS, ins), device=DEV, generator=g).float()
    w = mx.quantize_matrix(torch.randint(-2, 3, (outs, ins), device=DEV, generator=g).float(), mx.E2M1)
    y = mx.linear(w, mx.quantize_matrix(x, mx.E2M1), fn=mx.FN_RELU)
    for a, n in [(a, 32) for a in _blocks()] + [(ROWS // 32 * 32, ROWS % 32)]:
        part = mx.linear(w, mx.quantize_matrix(x[a:a + n].contiguous(), mx.E2M1), fn=mx.FN_RELU)
        assert torch.equal(y[a:a + n], part), a


def test_wgrad_reads_past_32_bits(mx):
    """dZ of 2.18e9 fp8 codes: the rows past the border count (integers, so
    every order of the sums is exact)."""
    outs, ins = 2080, 32
    dz = torch.zeros((ROWS, outs), dtype=torch.bfloat16, device=DEV)
    x = torch.ones((ROWS, ins), device=DEV)
    marks = [a + 7 for a in _blocks()] + [ROWS - 1]
    want = torch.zeros(outs, device=DEV)
    for k, r in enumerate(marks):
        dz[r, (5 + 97 * k) % outs] = 1 + k % 3
        want[(5 + 97 * k) % outs] += 1 + k % 3
    q = mx.quantize_matrix(dz, mx.E4M3)
    del dz
    dw, db = mx.linear_wgrad(q, mx.quantize_matrix(x, mx.E4M3))
    assert torch.equal(db, want)
    assert torch.equal(dw, want[:, None].expand(outs, ins))


def test_norm_past_32_bits(mx):
    d = 2080
    g = torch.Generator(DEV).manual_seed(3)
    x, y = (torch.empty((ROWS, d), dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(2))
    wp, wq = (torch.randn(d, device=DEV, generator=g) for _ in range(2))
    h, u = mx.norm_residual(x, y, w_post=wp, w_pre=wq, scale=0.5)
    for a in _blocks() + [ROWS - 32]:
        hh, uu = mx.norm_residual(x[a:a + 32].contiguous(), y[a:a + 32].contiguous(), w_post=wp, w_pre=wq, scale=0.5)
        assert torch.equal(h[a:a + 32], hh) and torch.equal(u[a:a + 32], uu), a
    del u
    dx, dy, *_ = mx.norm_residual_backward(x, y, h, y, w_post=wp, w_pre=wq, scale=0.5)
    for a in _blocks() + [ROWS - 32]:
        s = slice(a, a + 32)
        px, py, *_ = mx.norm_residual_backward(*(t[s].contiguous() for t in (x, y, h, y)), w_post=wp, w_pre=wq, scale=0.5)
        assert torch.equal(dx[s], px) and torch.equal(dy[s], py), a


def test_clip_past_32_bits(mx):
    n = (1 << 31) + 12345
    t = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    t[-1] = 3
    out = torch.zeros_like(t)
    norm = float(mx.grad_clip([t, t[:100]], 1.0, out=[out, torch.empty_like(t[:100])]))
    want = math.sqrt(n + 8 + 100)
    assert abs(norm - want) <= 2.0 ** -23 * want
    c = torch.tensor(1.0 / (want + 1e-6), dtype=torch.float32)
    assert out[0].item() == c.bfloat16().item() and out[(1 << 31) - 1].item() == out[1 << 31].item() == out[0].item()
    assert out[-1].item() == (3 * c).bfloat16().item() and int((out == 0).sum()) == 0
