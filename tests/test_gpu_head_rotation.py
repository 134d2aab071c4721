"""Position rotation of query and key heads, per-head norms and R_3 through the C ABI, against the float64 oracle.

Bounds.  An angle is off by at most 2^-26 of a turn (2^-23.3 rad), cosine, sine and the amplitude by three roundings more:
2^-22 m in all; the rotation adds two roundings of its terms: |error| <= 2^-21 m (|a| + |b|) for a pair (a, b).  R_3 preserves the 2-norm, which
these errors grow by at most 2 * 2^-21 m ||x||, and rounds log2(d) + 2 times: <= 2^-19 m ||x|| per element.  The norm's factor has about 25 roundings of a
sum of squares (half of them after the root) and four more: 2^-20 relative.  Together 2^-18 m ||x|| covers every forward element and the gradient
taken back; dx = r (w g - x r^2 mean(w g x)) has two terms of at most r max|w| ||g|| each: 2^-17 r max|w| m ||dy||.  A stored bf16 adds 2^-8 |y|."""
import numpy as np
import pytest

from oracle import heads_oracle as H

pytestmark = pytest.mark.gpu

SCALINGS = {
    "none": dict(),
    "linear": dict(scaling="linear", factor=8.0),
    "ntk": dict(scaling="ntk", factor=4.0),
    "bands": dict(theta=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192),
    "ramp": dict(scaling="ramp", factor=16.0, low=1.0, high=32.0, original=4096),
}


def _t():
    import torch
    return torch


def _B():
    from paper_2605_10793_b200 import binding as B
    return B


def _np(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def _data(seed, n, h, d, dtype, kind="fused"):
    """Head rows (n, h, d) inside a wider buffer: a slice of a fused projection, heads before tokens, or one element off."""
    torch = _t()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    if kind == "fused":
        x = torch.empty(n, h + 3, d, device="cuda", dtype=dt)[:, 1:1 + h]
    elif kind == "heads_first":
        x = torch.empty(h, n, d, device="cuda", dtype=dt).transpose(0, 1)
    else:
        x = torch.empty(n, h * d + 3, device="cuda", dtype=dt)[:, 1:1 + h * d].unflatten(1, (h, d))
    v = torch.randn(n, h, d, device="cuda", generator=g)
    v[..., d // 3] *= 20.0
    x.copy_(v * torch.exp(torch.randn(n, 1, 1, device="cuda", generator=g)))
    return x


def _positions(seed, n, far):
    torch = _t()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    p = torch.randint(0, far, (n,), device="cuda", generator=g)
    p[0] = 0
    return p


def _within(got, want, bound, dtype):
    bound = bound + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 2.0 ** -24 * np.abs(want)) + 1e-37
    bad = np.abs(got - want) > bound
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - want) / bound)))


def _norms(x):
    return np.linalg.norm(x, axis=-1, keepdims=True)


SHAPES = [(64, 64), (64, 32), (80, 80), (80, 40), (96, 32), (96, 24), (112, 112), (128, 128), (128, 64), (128, 32), (128, 48), (192, 192), (256, 256),
          (256, 96), (128, 0), (2, 2), (6, 4), (33, 10), (512, 512), (320, 320), (16, 16), (32, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,r", SHAPES)
def test_rotation_forward_and_inverse(d, r, layout, dtype):
    B, torch = _B(), _t()
    name = sorted(SCALINGS)[(d + r + (layout == "half")) % 5]
    if r == 2 and name == "ntk":
        name = "none"
    rope = B.Rope(r, layout=layout, **SCALINGS[name]) if r else None
    freq, amp = H.frequencies(r, **SCALINGS[name]) if r else (np.zeros(0), 1.0)
    n = 61
    q, k = _data(d, n, 5, d, dtype), _data(d + 1, n, 2, d, dtype)
    pos = _positions(d, n, 200000)
    for r3 in ([False, True] if d >= 4 and d & (d - 1) == 0 else [False]):
        yq, yk = B.conqur_rope_heads(q, k, pos, rope, hadamard=r3)
        zq, zk = B.conqur_rope_heads(q, k, pos, rope, hadamard=r3, inverse=True)
        for x, y, z in ((q, yq, zq), (k, yk, zk)):
            x64, p = _np(x), pos.cpu().numpy()
            bound = 2.0 ** -18 * amp * _norms(x64)
            _within(_np(y), H.norm_rotate(x64, None, 0.0, p, freq, amp, layout, r3), bound, dtype)
            _within(_np(z), H.rotate_inverse(x64, p, freq, amp, layout, r3), bound, dtype)


@pytest.mark.parametrize("kind", ["fused", "heads_first", "unaligned"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,r,layout,r3", [(128, 128, "half", True), (64, 32, "half", False), (96, 24, "half", False), (80, 80, "interleaved", False),
                                           (256, 64, "half", True), (8, 6, "half", True), (128, 96, "half", True), (48, 48, "half", False)])
def test_normed_heads_forward_and_gradients(d, r, layout, r3, dtype, kind):
    B, torch = _B(), _t()
    rope = B.Rope(r, layout=layout, **SCALINGS["ramp"])
    freq, amp = H.frequencies(r, **SCALINGS["ramp"])
    n, hq, hk, eps = 75, 7, 2, 1e-5
    q, k = _data(d, n, hq, d, dtype, kind), _data(d + 1, n, hk, d, dtype, kind)
    q[3] = 0                                                    # a row of zeros: its norm is sqrt(eps)
    gq, gk = _data(d + 2, n, hq, d, dtype, kind), _data(d + 3, n, hk, d, dtype, kind)
    w = [(1.0 + 0.3 * torch.randn(d, device="cuda")).to(q.dtype) for _ in range(2)]
    pos = _positions(d, n, 100000)
    y = B.conqur_norm_rope_heads(q, k, w[0], w[1], pos, rope, eps, hadamard=r3)
    grads = B.conqur_norm_rope_heads_backward(gq, gk, q, k, w[0], w[1], pos, rope, eps, hadamard=r3)
    again = B.conqur_norm_rope_heads_backward(gq, gk, q, k, w[0], w[1], pos, rope, eps, hadamard=r3)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    p = pos.cpu().numpy()
    for i, (x, g) in enumerate(((q, gq), (k, gk))):
        x64, w64, g64 = _np(x), _np(w[i]), _np(g)
        want = H.norm_rotate(x64, w64, eps, p, freq, amp, layout, r3)
        rms = 1.0 / np.sqrt(np.mean(x64 * x64, axis=-1, keepdims=True) + eps)
        _within(_np(y[i]), want, 2.0 ** -18 * amp * _norms(x64 * rms * w64), dtype)
        dx, dw = H.norm_rotate_grad(g64, x64, w64, eps, p, freq, amp, layout, r3)
        _within(_np(grads[i]), dx, 2.0 ** -17 * rms * np.max(np.abs(w64)) * amp * _norms(g64), dtype)
        # a sum over n * heads rows in at most 256 roundings (2^-16 of the terms' sum), of terms off by 2^-18 m ||dy|| |x r|
        terms = np.abs(x64 * rms) * amp * _norms(g64)
        _within(_np(grads[2 + i]), dw, (2.0 ** -16 + 2.0 ** -18) * terms.sum(axis=(0, 1)), "f32")


def test_gradients_against_differences():
    """The backward pass against central differences of the forward pass in fp32: a random direction of inputs and weights."""
    B, torch = _B(), _t()
    d, n, eps = 64, 9, 1e-3
    rope = B.Rope(32, layout="half")
    pos = _positions(1, n, 5000)
    q, k = (torch.randn(n, h, d, device="cuda") for h in (3, 1))
    wq, wk = (1.0 + 0.1 * torch.randn(d, device="cuda") for _ in range(2))
    gq, gk = (torch.randn(n, h, d, device="cuda") for h in (3, 1))
    dq, dk, dwq, dwk = B.conqur_norm_rope_heads_backward(gq, gk, q, k, wq, wk, pos, rope, eps, hadamard=True)
    dirs = [torch.randn_like(t) for t in (q, k, wq, wk)]
    step = 2.0 ** -6

    def loss(s):
        a, b, u, v = (t + s * e for t, e in zip((q, k, wq, wk), dirs))
        yq, yk = B.conqur_norm_rope_heads(a, b, u, v, pos, rope, eps, hadamard=True)
        return float((yq.double() * gq).sum() + (yk.double() * gk).sum())

    # four-point difference: the error term is step^4 / 30 of the fifth derivative (the map is smooth on the scale of its rows' rms,
    # about 1: derivatives of the order of the terms' sum), 2^-24 rounding of 36 rows' sums over 2 step
    numeric = (8 * (loss(step) - loss(-step)) - (loss(2 * step) - loss(-2 * step))) / (12 * step)
    formula = sum(float((a.double() * b).sum()) for a, b in zip((dq, dk, dwq, dwk), dirs))
    size = sum(float((a.double() * b).abs().sum()) for a, b in zip((dq, dk, dwq, dwk), dirs))
    assert abs(numeric - formula) <= 1e-4 * size, (numeric, formula, size)


def test_far_negative_and_largest_positions():
    """Angles are exact modulo a turn at any int64 position; pairs keep their length."""
    B, torch = _B(), _t()
    d = 128
    far = [0, 1, -1, 2 ** 20 + 1, 2 ** 31, 2 ** 40 + 12345, -2 ** 40 - 7, 2 ** 62 + 1]
    pos = torch.tensor(far, device="cuda")
    x = torch.randn(len(far), 2, d, device="cuda")
    rope = B.Rope(d, layout="half")
    y, _ = B.conqur_rope_heads(x, None, pos, rope)
    back, _ = B.conqur_rope_heads(y, None, pos, rope, inverse=True)
    assert (back - x).abs().max().item() <= 2.0 ** -19 * float(x.norm(dim=-1).max())
    # the table's own frequencies (64-bit fractions of a turn), in whole numbers
    words = [int(v) & (2 ** 64 - 1) for v in rope.table[: d // 2].tolist()]
    turn = np.array([[((p * w) & (2 ** 64 - 1)) / 2.0 ** 64 for w in words] for p in far])
    c, s = np.cos(2 * np.pi * turn)[:, None], np.sin(2 * np.pi * turn)[:, None]
    x64 = _np(x)
    a, b = x64[..., : d // 2], x64[..., d // 2:]
    _within(_np(y), np.concatenate((a * c - b * s, a * s + b * c), axis=-1), 2.0 ** -18 * _norms(x64), "f32")
    # and these are the frequencies of the definition, to 2^-60 of a turn
    freq, _ = H.frequencies(d)
    assert np.max(np.abs(np.array(words, dtype=np.float64) / 2.0 ** 64 - freq / (2 * np.pi))) <= 2.0 ** -52


def test_layouts_batches_in_place_streams_and_graphs():
    B, torch = _B(), _t()
    d, b, t = 128, 3, 17
    rope = B.Rope(d, layout="half", **SCALINGS["bands"])
    q = torch.randn(b, t, 6, d, device="cuda").bfloat16()
    k = torch.randn(b, 2, t, d, device="cuda").bfloat16().transpose(1, 2)      # heads before tokens
    pos = torch.randint(0, 9000, (b, t), device="cuda")
    yq, yk = B.conqur_rope_heads(q, k, pos, rope, hadamard=True)
    fq, fk = B.conqur_rope_heads(q.flatten(0, 1), k.contiguous().flatten(0, 1), pos.flatten(), rope, hadamard=True)
    assert torch.equal(yq.flatten(0, 1), fq) and torch.equal(yk.flatten(0, 1), fk)
    # one row of positions for every sequence
    same = pos[:1].expand(b, t)
    assert torch.equal(B.conqur_rope_heads(q, None, pos[0], rope)[0], B.conqur_rope_heads(q, None, same, rope)[0])
    assert torch.equal(B.conqur_rope_heads(q, None, pos[0], rope)[0], B.conqur_rope_heads(q, None, same.contiguous(), rope)[0])
    # in place inside a fused buffer: the values beside the heads stay
    buf = torch.randn(b * t, 10, d, device="cuda").bfloat16()
    old = buf.clone()
    want = B.conqur_rope_heads(buf[:, :6], buf[:, 6:8], pos.flatten(), rope, hadamard=True)
    B.conqur_rope_heads(buf[:, :6], buf[:, 6:8], pos.flatten(), rope, hadamard=True, out=(buf[:, :6], buf[:, 6:8]))
    assert torch.equal(buf[:, :6], want[0]) and torch.equal(buf[:, 6:8], want[1]) and torch.equal(buf[:, 8:], old[:, 8:])
    # keys shared by their heads (stride 0 in, rows of their own out)
    one = torch.randn(t, 1, d, device="cuda")
    many, _ = B.conqur_rope_heads(one.expand(t, 4, d), None, pos[0], rope)
    assert all(torch.equal(many[:, h], B.conqur_rope_heads(one, None, pos[0], rope)[0][:, 0]) for h in range(4))
    # another stream, captured and replayed on new contents
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = (torch.empty_like(yq), torch.empty(k.shape, dtype=k.dtype, device="cuda"))
        B.conqur_rope_heads(q, k, pos, rope, hadamard=True, out=out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out[0], yq) and torch.equal(out[1], yk)
    w = torch.ones(d, device="cuda")
    graph = torch.cuda.CUDAGraph()
    gy = torch.randn_like(q)
    gk = torch.randn(k.shape, device="cuda").bfloat16()
    qs, ks = q.clone(), k.clone()
    B.conqur_norm_rope_heads_backward(gy, gk, qs, ks, w, w, pos, rope)
    with torch.cuda.graph(graph):
        fwd = B.conqur_norm_rope_heads(qs, ks, w, w, pos, rope)
        bwd = B.conqur_norm_rope_heads_backward(gy, gk, qs, ks, w, w, pos, rope)
    qs.copy_(q.flip(0))
    ks.copy_(k.flip(0))
    graph.replay()
    assert all(torch.equal(a, c) for a, c in zip(fwd, B.conqur_norm_rope_heads(qs, ks, w, w, pos, rope)))
    assert all(torch.equal(a, c) for a, c in zip(bwd, B.conqur_norm_rope_heads_backward(gy, gk, qs, ks, w, w, pos, rope)))


def test_values_that_are_not_finite_stay_in_their_row_and_pair():
    B, torch = _B(), _t()
    d = 128
    rope = B.Rope(64, layout="half")
    pos = torch.arange(8, device="cuda") + 5
    for dt in (torch.float32, torch.bfloat16):
        x = torch.randn(8, 4, d, device="cuda").to(dt)
        clean, _ = B.conqur_rope_heads(x, None, pos, rope)
        x[2, 1, 3], x[5, 3, 100] = float("nan"), float("inf")
        y, _ = B.conqur_rope_heads(x, None, pos, rope)
        hit = torch.zeros_like(x, dtype=torch.bool)
        hit[2, 1, [3, 35]] = True
        hit[5, 3, 100] = True
        assert torch.equal(y[~hit], clean[~hit]) and torch.isnan(y[2, 1, [3, 35]]).all() and torch.isinf(y[5, 3, 100])
        n, _ = B.conqur_norm_rope_heads(x, None, None, None, pos, rope)
        rows = torch.isfinite(n).all(dim=-1)
        rows[2, 1] = rows[5, 3] = True
        assert rows.all() and torch.isnan(n[2, 1]).all()


@pytest.mark.parametrize("n", [0, 1, 2, 700])
def test_token_counts_and_single_tensors(n):
    B, torch = _B(), _t()
    d = 64
    rope = B.Rope(d, layout="interleaved")
    pos = torch.arange(n, device="cuda")
    q = torch.randn(n, 3, d, device="cuda")
    y, none = B.conqur_rope_heads(q, None, pos, rope)
    assert none is None and y.shape == q.shape
    g = torch.randn_like(q)
    w = torch.ones(d, device="cuda")
    dq, dk, dwq, dwk = B.conqur_norm_rope_heads_backward(g, None, q, None, w, None, pos, rope)
    assert dk is None and dwk is None
    if n == 0:
        assert not dwq.any().item()
        return
    freq, amp = H.frequencies(d)
    want, dw = H.norm_rotate_grad(_np(g), _np(q), np.ones(d), 1e-6, pos.cpu().numpy(), freq, amp, "interleaved", False)
    _within(_np(dq), want, 2.0 ** -17 * _norms(_np(g)) / np.sqrt(np.mean(_np(q) ** 2, axis=-1, keepdims=True)), "f32")
    _within(_np(y), H.norm_rotate(_np(q), None, 0, pos.cpu().numpy(), freq, amp, "interleaved", False), 2.0 ** -18 * _norms(_np(q)), "f32")


def test_sizes_past_32_bit_offsets():
    """Element offsets beyond 2^32: the last tokens of a 9 GB buffer are rotated like a small copy of them."""
    B, torch = _B(), _t()
    d, h = 128, 8
    n = (2 ** 32) // (h * d) + 300
    x = torch.zeros(n, h, d, dtype=torch.bfloat16, device="cuda")
    x[-70:].normal_()
    x[:70].normal_()
    pos = torch.arange(n, device="cuda")
    rope = B.Rope(d)
    B.conqur_rope_heads(x[-70:].clone(), None, pos[-70:], rope)
    for part in (slice(0, 70), slice(n - 70, n)):
        want, _ = B.conqur_rope_heads(x[part].clone(), None, pos[part].clone(), rope)
        if part.start == 0:
            first = want
        else:
            last = want
    B.conqur_rope_heads(x, None, pos, rope, out=(x, None))
    assert torch.equal(x[:70], first) and torch.equal(x[-70:], last) and not x[70:-70:1013].any().item()
