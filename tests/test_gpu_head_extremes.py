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


def _turns(r, theta=10000.0, scaling="none", factor=1.0, low=0.0, high=0.0, original=0):
    """The frequencies in turns per position, to 50 digits (amplitudes aside)."""
    from decimal import ROUND_CEILING, ROUND_FLOOR, Decimal as D, getcontext
    getcontext().prec = 60
    tau = 2 * D("3.14159265358979323846264338327950288419716939937510582097494459")
    base, factor, out = D(theta).ln(), D(factor), []
    if scaling == "ntk":
        base += factor.ln() * r / (r - 2)
    for i in range(r // 2):
        f = (-base * 2 * i / r).exp()
        if scaling == "linear":
            f /= factor
        elif scaling == "bands":
            keep = min(max((D(original) * f / tau - D(low)) / (D(high) - D(low)), D(0)), D(1))
            f *= keep + (1 - keep) / factor
        elif scaling == "ramp":
            dim = lambda u: r * (D(original) / (tau * D(u))).ln() / (2 * base)       # noqa: E731
            a = max(dim(high).to_integral_value(ROUND_FLOOR), D(0))
            b = min(dim(low).to_integral_value(ROUND_CEILING), D(r - 1))
            g = min(max((i - a) / max(b - a, D("0.001")), D(0)), D(1))
            f = f * (1 - g) + f / factor * g
        out.append(f / tau)
    return out


@pytest.mark.parametrize("name", sorted(SCALINGS))
@pytest.mark.parametrize("r", [4, 64, 128, 512])
def test_frequencies_are_held_to_the_last_of_64_bits(r, name):
    """A frequency's 64-bit fraction of a turn is off by less than one unit (2^-64): what positions multiply.  Against 60-digit arithmetic."""
    from decimal import Decimal as D
    B = _B()
    for theta in ([10000.0, 1e6] if name not in ("bands", "ramp") else [SCALINGS[name].get("theta", 10000.0)]):
        kw = dict(SCALINGS[name], theta=theta)
        words = [int(v) & (2 ** 64 - 1) for v in B.Rope(r, **kw).table[: r // 2].tolist()]
        for w, f in zip(words, _turns(r, **kw)):
            assert abs(D(w) - f * D(2) ** 64) < 1


@pytest.mark.parametrize("name", ["none", "bands"])
def test_far_positions_against_the_frequencies_of_the_definition(name):
    """Angles are off by at most |position| 2^-64 + 2^-26 of a turn."""
    from decimal import Decimal as D
    B, torch = _B(), _t()
    d = 128
    rope = B.Rope(d, layout="half", **SCALINGS[name])
    far = [0, 7, 200000, 2 ** 31 - 1, 2 ** 31 + 5, -2 ** 31 - 5, 2 ** 36 + 99, 2 ** 40 + 12345, -2 ** 40 - 7, 2 ** 44 + 1]
    turns = [[p * f for f in _turns(d, **SCALINGS[name])] for p in far]
    turn = np.array([[float(t - t.to_integral_value()) for t in row] for row in turns])
    x = torch.randn(len(far), 2, d, device="cuda")
    y, _ = B.conqur_rope_heads(x, None, torch.tensor(far, device="cuda"), rope)
    c, s = np.cos(2 * np.pi * turn)[:, None], np.sin(2 * np.pi * turn)[:, None]
    x64 = _np(x)
    a, b = x64[..., : d // 2], x64[..., d // 2:]
    want = np.concatenate((a * c - b * s, a * s + b * c), axis=-1)
    word = 2 * np.pi * np.abs(np.array(far, dtype=np.float64))[:, None, None] * 2.0 ** -64
    _within(_np(y), want, (2.0 ** -18 + word) * _norms(x64), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,r,layout", [(128, 64, "half"), (80, 40, "interleaved"), (96, 24, "half")])
def test_backward_in_place_and_with_a_scratch_of_the_caller(d, r, layout, dtype):
    """The gradients of the inputs may take the place of those of the outputs (or of the inputs), inside a wider buffer; the scratch may hold anything."""
    B, torch = _B(), _t()
    rope = B.Rope(r, layout=layout)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, hq, hk = 301, 6, 2
    x = torch.randn(n, hq + hk + 1, d, device="cuda").to(dt)
    g = torch.randn(n, hq + hk + 1, d, device="cuda").to(dt)
    split = lambda t: (t[:, :hq], t[:, hq:hq + hk])                            # noqa: E731
    w = [(1.0 + 0.3 * torch.randn(d, device="cuda")).to(dt) for _ in range(2)]
    pos = torch.arange(n, device="cuda") + 17
    want = B.conqur_norm_rope_heads_backward(*split(g), *split(x), *w, pos, rope, hadamard=d == 128)
    scratch = torch.full((B.load().conqur_norm_rope_backward_scratch_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    for own in (g.clone(), None):
        grads, heads = (own, x) if own is not None else (g, x.clone())
        into = grads if own is not None else heads
        got = B.conqur_norm_rope_heads_backward(*split(grads), *split(heads), *w, pos, rope, hadamard=d == 128, out=split(into), scratch=scratch)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert got[0].data_ptr() == into.data_ptr() and torch.equal(into[:, -1], (g if own is not None else x)[:, -1])
    with pytest.raises(B.ConqurError):
        B.conqur_norm_rope_heads_backward(*split(g), *split(x), *w, pos, rope, scratch=scratch[:-256])
    with pytest.raises(B.ConqurError):
        B.conqur_norm_rope_heads_backward(*split(g), *split(x), *w, pos, rope, scratch=torch.empty(scratch.numel() + 64, dtype=torch.uint8, device="cuda")[8:])


def test_backward_past_32_bit_offsets():
    """Element offsets beyond 2^32: the first and last tokens' gradients are those of small copies; the weight gradients are both ends' sums."""
    B, torch = _B(), _t()
    d, h = 128, 8
    n = (2 ** 32) // (h * d) + 300
    x = torch.zeros(n, h, d, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros_like(x)
    ends = (slice(0, 70), slice(n - 70, n))
    for e in ends:
        x[e].normal_()
        g[e].normal_()
    pos = torch.arange(n, device="cuda")
    w = (1.0 + 0.3 * torch.randn(d, device="cuda")).bfloat16()
    rope = B.Rope(d)
    small = [B.conqur_norm_rope_heads_backward(g[e].clone(), None, x[e].clone(), None, w, None, pos[e].clone(), rope) for e in ends]
    x64, g64 = (np.concatenate([_np(t[e]) for e in ends]) for t in (x, g))
    rms = 1.0 / np.sqrt(np.mean(x64 * x64, axis=-1, keepdims=True) + 1e-6)
    dq, _, dw, _ = B.conqur_norm_rope_heads_backward(g, None, x, None, w, None, pos, rope, out=(g, None))
    assert all(torch.equal(dq[e], s[0]) for e, s in zip(ends, small)) and not dq[70:-70:1013].any().item()
    bound = 2 * (2.0 ** -16 + 2.0 ** -18) * (np.abs(x64 * rms) * _norms(g64)).sum(axis=(0, 1))
    _within(_np(dw), _np(small[0][2]) + _np(small[1][2]), bound, "f32")
