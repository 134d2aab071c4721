"""Normed heads at the ends of the range, and calls of the backward pass that share memory, against the float64 oracle (bounds: test_gpu_head_rotation.py)."""
import numpy as np
import pytest

from oracle import heads_oracle as H
from tests.test_gpu_head_rotation import SCALINGS, _B, _np, _norms, _positions, _t, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,r,layout,r3", [(128, 128, "half", True), (128, 64, "interleaved", True), (64, 32, "half", False), (256, 64, "half", True),
                                           (80, 80, "interleaved", False), (112, 112, "half", False), (96, 24, "half", False), (8, 6, "half", True)])
def test_rows_whose_squares_pass_an_fp32(d, r, layout, r3, dtype):
    """A norm takes any row's size off, also that of rows from 2e19 on, whose squares are more than an fp32 holds; their neighbours keep their bits."""
    B, torch = _B(), _t()
    rope = B.Rope(r, layout=layout, **SCALINGS["ramp"])
    freq, amp = H.frequencies(r, **SCALINGS["ramp"])
    n, hq, hk, eps = 75, 7, 2, 1e-5
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d + r)
    rand = lambda h: torch.randn(n, h, d, device="cuda", generator=gen)       # noqa: E731
    sizes = torch.tensor([1.0, 1e18, 1e20, 1e30, 3e36], device="cuda")
    scale = [sizes[torch.randint(0, 5, (n, h, 1), device="cuda", generator=gen)] for h in (hq, hk)]
    plain = [rand(hq), rand(hk)]
    q, k = ((x * s).to(dt) for x, s in zip(plain, scale))
    gq, gk = rand(hq).to(dt), rand(hk).to(dt)
    w = [(1.0 + 0.3 * torch.randn(d, device="cuda", generator=gen)).to(dt) for _ in range(2)]
    pos = _positions(d, n, 100000)
    y = B.conqur_norm_rope_heads(q, k, w[0], w[1], pos, rope, eps, hadamard=r3)
    grads = B.conqur_norm_rope_heads_backward(gq, gk, q, k, w[0], w[1], pos, rope, eps, hadamard=r3)
    p = pos.cpu().numpy()
    for i, (x, g) in enumerate(((q, gq), (k, gk))):
        x64, w64, g64 = _np(x), _np(w[i]), _np(g)
        rms = 1.0 / np.sqrt(np.mean(x64 * x64, axis=-1, keepdims=True) + eps)
        _within(_np(y[i]), H.norm_rotate(x64, w64, eps, p, freq, amp, layout, r3), 2.0 ** -18 * amp * _norms(x64 * rms * w64), dtype)
        dx, dw = H.norm_rotate_grad(g64, x64, w64, eps, p, freq, amp, layout, r3)
        _within(_np(grads[i]), dx, 2.0 ** -17 * rms * np.max(np.abs(w64)) * amp * _norms(g64), dtype)
        terms = np.abs(x64 * rms) * amp * _norms(g64)
        _within(_np(grads[2 + i]), dw, (2.0 ** -16 + 2.0 ** -18) * terms.sum(axis=(0, 1)), "f32")
    # rows of ordinary size beside them: as without them
    q1, k1 = ((x * torch.where(s == 1.0, s, torch.ones_like(s))).to(dt) for x, s in zip(plain, scale))
    y1 = B.conqur_norm_rope_heads(q1, k1, w[0], w[1], pos, rope, eps, hadamard=r3)
    g1 = B.conqur_norm_rope_heads_backward(gq, gk, q1, k1, w[0], w[1], pos, rope, eps, hadamard=r3)
    for i in range(2):
        same = (scale[i] == 1.0)[..., 0]
        assert torch.equal(y[i][same], y1[i][same]) and torch.equal(grads[i][same], g1[i][same])
