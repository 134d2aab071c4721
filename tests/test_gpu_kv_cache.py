"""The paged cache and the attention over it through the C ABI, against the float64 oracle.

The cache's codes are exact: the step is rounded to bf16 before it divides, ties are ties (byte for byte against the oracle).

Attention's bounds, per element of a row with probabilities p_l and largest sum of |q k| scale over the positions S: a score is a sum of d
exact products in fp32, 16 at a time, which leaves at most 2^-18 S with its scaling (delta); exponentials and sums add 2^-20; a probability is rounded to bf16
before it meets the values (2^-8): |error| <= (2^-8 + 2 delta + 2^-19) sum p |v| + 2^-8 |out|.  With 4 bits the products hold codes, not
code - zero-point: sums of up to 15 sum p step, rounded (or cut, 2^-23) once per 16 tokens of one of eight warps and in some 12 additions of parts, less sum p
zero-point step: (positions / 128 + 12) 2^-23 15 sum p step more.  lse: delta, 2^-20 of its size and the rounding of a sum of up to
2^11 terms a lane, 2^-13."""
import numpy as np
import pytest

from oracle import kv_oracle as K

pytestmark = pytest.mark.gpu


def _t():
    import torch
    return torch


def _B():
    from paper_2605_10793_b200 import binding as B
    return B


def _rows(seed, *shape):
    """bf16 rows whose quotients by a step are often ties: small whole multiples beside ordinary values."""
    r = np.random.default_rng(seed)
    x = r.standard_normal(shape) * np.exp(r.standard_normal(shape[:-1] + (1,)))
    tie = r.random(shape[:-1]) < 0.5
    x[tie] = np.round(4 * x[tie]) * 0.5
    x.reshape(-1, shape[-1])[0] = 0.0
    x.reshape(-1, shape[-1])[-1] = np.abs(x.reshape(-1, shape[-1])[-1]) + 1.0
    x.reshape(-1, shape[-1])[x.size // shape[-1] // 2] = -3.25
    return K.bf16(x)


def _dev(x):
    torch = _t()
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.float32)).cuda().bfloat16()


@pytest.mark.parametrize("n", [1, 5, 77])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits,clip", [(4, 1.0), (4, 0.9), (16, 1.0)])
def test_append_writes_the_documented_bytes_and_read_gives_their_values(bits, clip, d, page, n):
    B, torch = _B(), _t()
    heads, pages = 3, 7
    r = np.random.default_rng(n * page + d)
    slots = r.permutation(pages * page)[:n]
    if n > 2:
        slots[[1, n // 2]] = -1
    k, v = _rows(n + d, n, heads, d), _rows(n + d + 1, n, heads, d)
    cache = B.KVCache(pages, page, heads, d, bits=bits, clip_ratio=clip, data=torch.full((pages, heads, K.block_bytes(page, d, bits)), 0xA5, dtype=torch.uint8, device="cuda"))
    s = torch.from_numpy(slots).cuda()
    B.conqur_kv_append(cache, _dev(k), _dev(v), s)
    # whole blocks by the oracle, of which the bytes of the stored tokens count
    want = np.full((pages, heads, K.block_bytes(page, d, bits)), 0xA5, np.uint8)
    for p in range(pages):
        place = {int(x) % page: i for i, x in enumerate(slots) if x >= 0 and x // page == p}
        for h in range(heads):
            kk, vv = np.zeros((page, d)), np.zeros((page, d))
            for t, i in place.items():
                kk[t], vv[t] = k[i, h], v[i, h]
            block = K.pack(kk, vv, page, bits, clip)
            mine = np.zeros(block.shape, bool)
            for t in place:
                if bits == 4:
                    for base, w in ((0, d // 2), (page * d // 2, d // 2), (page * d, 4), (page * d + 4 * page, 4)):
                        mine[base + t * w:base + (t + 1) * w] = True
                else:
                    for plane in range(2 * d // 64):
                        mine[(plane * page + t) * 128:(plane * page + t + 1) * 128] = True
            want[p, h][mine] = block[mine]
    assert np.array_equal(cache.data.cpu().numpy(), want)
    kr, vr = B.conqur_kv_read(cache, s, torch.float32)
    kb, vb = B.conqur_kv_read(cache, s)
    stored = (slots >= 0)[:, None, None]
    for got, half, y in ((kr, kb, k), (vr, vb, v)):
        val = np.where(stored, K.values(y, bits, clip), 0.0)
        assert np.array_equal(got.cpu().numpy().astype(np.float64), val)
        assert np.array_equal(half.float().cpu().numpy().astype(np.float64), K.bf16(val))
    assert B.conqur_kv_status() == 0


def test_every_tie_and_step_rounds_like_the_definition():
    """All pairs of a step's significand and a value's: rows of one range end and all multiples near ties, every exponent apart up to 2^-20."""
    B, torch = _B(), _t()
    sig = np.arange(128, 256)
    rows = []
    for top in sig[::3]:
        y = np.concatenate([np.array([top * 15 * 2.0 ** -4, -top * 2.0 ** (top % 5 - 4)]), sig[top % 2::4] * 2.0 ** (top % 7 - 9), -sig[top % 3::4] * 2.0 ** (top % 6 - 11)])
        rows.append(np.resize(y, 128))
    y = K.bf16(np.array(rows))[:, None, :]
    y = np.concatenate([y, y * 2.0 ** -60, y * 2.0 ** 90, y * 2.0 ** -110, -y], axis=0)
    y = K.bf16(y)
    n = y.shape[0]
    cache = B.KVCache(n // 16 + 1, 16, 1, 128)
    s = torch.arange(n, device="cuda")
    B.conqur_kv_append(cache, _dev(y), _dev(-y), s)
    k, v = B.conqur_kv_read(cache, s, torch.float32)
    assert np.array_equal(k.cpu().numpy().astype(np.float64), K.values(y, 4))
    assert np.array_equal(v.cpu().numpy().astype(np.float64), K.values(-y, 4))


def test_append_odd_layouts_extremes_and_bad_slots():
    B, torch = _B(), _t()
    n, heads, d, page = 40, 2, 128, 16
    wide = torch.randn(n, heads * d + 3, device="cuda").bfloat16()
    k = wide[:, 1:1 + heads * d].unflatten(1, (heads, d))                       # rows off 16-byte boundaries
    v = torch.randn(heads, n, d, device="cuda").bfloat16().transpose(0, 1)      # heads before tokens
    a, b = (B.KVCache(3, page, heads, d, data=torch.zeros(3, heads, K.block_bytes(page, d, 4), dtype=torch.uint8, device="cuda")) for _ in range(2))
    s = torch.arange(n, device="cuda") + 2
    B.conqur_kv_append(a, k, v, s)
    B.conqur_kv_append(b, k.contiguous(), v.contiguous(), s)
    assert torch.equal(a.data, b.data)
    # one row for all heads
    B.conqur_kv_append(a, k[:, :1].expand(n, heads, d), v[:, 1:].expand(n, heads, d), s)
    kr, vr = B.conqur_kv_read(a, s)
    assert torch.equal(kr[:, 0], kr[:, 1]) and torch.equal(vr[:, 0], vr[:, 1])
    # values that are not finite: their row reads NaN, the others stay
    bad = k.contiguous().clone()
    bad[3, 0, 5], bad[7, 1, 9], bad[9, 1, 0] = float("nan"), float("inf"), float("-inf")
    B.conqur_kv_append(b, bad, v.contiguous(), s)
    got, _ = B.conqur_kv_read(b, s)
    ref = torch.from_numpy(K.values(k.float().cpu().numpy().astype(np.float64), 4)).cuda()
    hit = torch.zeros(n, heads, dtype=torch.bool, device="cuda")
    hit[3, 0] = hit[7, 1] = hit[9, 1] = True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], ref.bfloat16()[~hit])
    # largest and smallest values: from 2^127 on a code's value might pass the largest fp32 (-8 steps of a range of 15 from -3.39e38 to 3.39e38 are -3.6e38)
    big = torch.full((1, heads, d), 3.3895313892515355e38, device="cuda").bfloat16()
    big[..., ::2] *= -1
    tiny = torch.full((1, heads, d), 2.0 ** -130, device="cuda").bfloat16()
    large = big * 0.5
    B.conqur_kv_append(b, torch.cat((big, tiny, large)), torch.cat((tiny, large, big)), s[:3])
    kk, vv = B.conqur_kv_read(b, s[:3], torch.float32)
    assert torch.isnan(kk[0]).all() and not kk[1].any() and not vv[0].any() and torch.isnan(vv[2]).all()
    assert torch.isfinite(kk[2]).all() and (kk[2].abs() > 1.5e38).all() and torch.equal(kk[2], vv[1])
    # slots beyond the cache are left out and told of; nothing is written outside
    guard = torch.full((5, heads, K.block_bytes(page, d, 4)), 0x5A, dtype=torch.uint8, device="cuda")
    c = B.KVCache(3, page, heads, d, data=guard[1:4])
    assert B.conqur_kv_status() == 0
    B.conqur_kv_append(c, k, v, torch.where(s % 2 == 0, s + 3 * page, -s))
    assert B.conqur_kv_status() == -11 and B.conqur_kv_status() == 0
    assert (guard == 0x5A).all()
    z, _ = B.conqur_kv_read(c, s + 3 * page)
    assert not z.any() and B.conqur_kv_status() == -11
    B.conqur_kv_append(c, k[:0], v[:0], s[:0])
    assert B.conqur_kv_read(c, s[:0])[0].shape == (0, heads, d)


# ---------------------------------------------------------------------------------------------------------- attention

def _tree_masks(rng, nodes, kind):
    out = []
    for n in nodes:
        m = [0] * n
        for j in range(n):
            parent = j - 1 if kind == "chain" else int(rng.integers(max(0, j - 3), j)) if j else -1
            m[j] = (m[parent] if parent >= 0 else 0) | (1 << j)
        if kind == "holes":
            m = [x if i % 3 else 0 for i, x in enumerate(m)]               # some see no drafted token, not even themselves
        out.append(m)
    return out


def _codes_bound(step, k, q, seen, scale):
    """What the sums of codes may add (see above); step (positions,), zeros where the cache holds bf16."""
    w = K.attend(q, k, step[:, None], seen, scale)[0]
    return (len(step) / 128 + 12) * 2.0 ** -23 * 15 * w


class Setup:
    """A batch of sequences whose keys and values lie in scattered pages; q packed with spare rows behind."""

    def __init__(self, seed, contexts, nodes, hk, group, d, page, bits, kind="tree", sharp=1.5):
        B, torch = _B(), _t()
        r = np.random.default_rng(seed)
        self.contexts, self.nodes, self.hk, self.group, self.d, self.page, self.bits = contexts, nodes, hk, group, d, page, bits
        lengths = [c + n for c, n in zip(contexts, nodes)]
        need = [-(-x // page) for x in lengths]
        pages = sum(need) + 2
        width = max(need + [1])
        order = r.permutation(pages)
        table = np.full((len(contexts), width), -1, np.int32)              # entries that no position needs may be anything
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.data = torch.full((pages, hk, K.block_bytes(page, d, bits)), 0xFF, dtype=torch.uint8, device="cuda")   # reads as NaN where nothing was written
        self.cache = B.KVCache(pages, page, hk, d, bits=bits, data=self.data)
        self.k, self.v, self.step = [], [], []
        for b, n in enumerate(lengths):
            k, v = K.bf16(r.standard_normal((n, hk, d))), K.bf16(r.standard_normal((n, hk, d)))
            k[..., : d // 16] = K.bf16(k[..., : d // 16] * 3)
            slots = np.array([table[b, l // page] * page + l % page for l in range(n)], dtype=np.int64).reshape(-1)
            if n:
                B.conqur_kv_append(self.cache, _dev(k), _dev(v), torch.from_numpy(slots).cuda())
            self.k.append(K.values(k, bits) if n else k)
            self.v.append(K.values(v, bits) if n else v)
            self.step.append(K.quantise(v)[2][..., 0] if n and bits == 4 else np.zeros((n, hk)))
        self.masks = _tree_masks(r, nodes, kind)
        self.starts = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        rows = int(self.starts[-1]) + 2
        self.q = K.bf16(sharp * r.standard_normal((rows, hk * group, d)))
        flat = [m for seq in self.masks for m in seq] + [0, 0]
        self.dev = dict(q=_dev(self.q), starts=torch.from_numpy(self.starts).cuda(), contexts=torch.tensor(contexts, dtype=torch.int32, device="cuda"),
                        table=torch.from_numpy(table).cuda())
        self.mask = torch.from_numpy(np.array(flat, dtype=np.uint64).view(np.int64)).cuda()
        self.rows = rows
        self.out = torch.full((rows, hk * group, d), 7.0, device="cuda").bfloat16()
        self.lse = torch.full((rows, hk * group), 7.0, device="cuda")

    def run(self, chain=False, **kw):
        B = _B()
        args = dict(max_nodes=max(self.nodes + [1]), out=self.out, lse=self.lse)
        args.update(kw)
        return B.conqur_tree_attention(self.dev["q"], self.cache, self.dev["starts"], self.dev["contexts"], self.dev["table"], None if chain else self.mask, **args)

    def check(self, out, lse, scale=None, chain=False):
        scale = self.d ** -0.5 if scale is None else scale
        o, l = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        for b, (c, n) in enumerate(zip(self.contexts, self.nodes)):
            if n == 0:
                continue
            a = self.starts[b]
            seen = np.zeros((n, c + n), bool)
            seen[:, :c] = True
            for i in range(n):
                for j in range(n):
                    seen[i, c + j] = j <= i if chain else (self.masks[b][i] >> j) & 1
            for h in range(self.hk * self.group):
                kh = h // self.group
                want, wl, mass, size = K.attend(self.q[a:a + n, h], self.k[b][:, kh], self.v[b][:, kh], seen, scale)
                delta = 2.0 ** -18 * size
                bound = (2.0 ** -8 + 2 * delta[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want) + 1e-30 + _codes_bound(self.step[b][:, kh], self.k[b][:, kh], self.q[a:a + n, h], seen, scale)
                err = np.abs(o[a:a + n, h] - want)
                assert (err <= bound).all(), (b, h, float((err / bound).max()))
                none = np.isneginf(wl)
                assert np.array_equal(none, np.isneginf(l[a:a + n, h]))
                ok = ~none
                assert (np.abs(l[a:a + n, h][ok] - wl[ok]) <= (delta + 2.0 ** -20 * np.abs(wl) + 2.0 ** -13)[ok]).all()
        # rows behind the last sequence
        assert (out[self.starts[-1]:] == 7.0).all() and (lse[self.starts[-1]:] == 7.0).all()


LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1027]


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hk,group,most,page", [(2, 1, 1, 16), (3, 4, 1, 64), (1, 8, 1, 32), (2, 5, 2, 16), (2, 16, 1, 64), (1, 4, 7, 32), (2, 7, 3, 16), (1, 8, 8, 64),
                                                (2, 4, 32, 16), (1, 3, 64, 32), (1, 16, 20, 64)])
def test_attention_over_all_row_counts_and_lengths(hk, group, most, page, d, bits):
    rng = np.random.default_rng(group * most + d)
    nodes = [most] + [int(rng.integers(0, most + 1)) for _ in LENGTHS[1:]]
    s = Setup(group + most, LENGTHS, nodes, hk, group, d, page, bits, "tree")
    s.check(*s.run())
    assert _B().conqur_kv_status() == 0


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("kind", ["chain", "holes"])
def test_masks_chains_and_rows_that_see_nothing(kind, bits):
    s = Setup(5, [0, 0, 3, 200], [4, 9, 9, 5], 2, 2, 128, 16, bits, kind, sharp=4.0)
    out, lse = s.run()
    s.check(out, lse)
    if kind == "holes":
        assert not out[0].any() and (lse[0] == float("-inf")).all()
    else:
        o2, l2 = s.run(chain=True, out=s.out.clone(), lse=s.lse.clone())
        assert _t().equal(o2, out) and _t().equal(l2, lse)
    out, lse = s.run(scale=-0.7)
    s.check(out, lse, scale=-0.7)
    out, lse = s.run(scale=0.0)
    s.check(out, lse, scale=0.0)


@pytest.mark.parametrize("bits", [4, 16])
def test_one_long_sequence_is_split_and_joined(bits):
    """Far more tiles than one CTA takes: the parts are added up; the same call gives the same bits, also through one workspace again and again."""
    B, torch = _B(), _t()
    s = Setup(11, [20000], [2], 2, 4, 128, 64, bits)
    ws = B.attention_workspace(s.cache, 4, 2)
    out, lse = s.run(workspace=ws)
    s.check(out, lse)
    for _ in range(5):
        o2, l2 = s.run(workspace=ws, out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0))
        assert torch.equal(o2, out) and torch.equal(l2, lse)
    # a larger workspace serves other sizes in between
    big = B.attention_workspace(s.cache, 16, 64)
    t = Setup(12, [500, 40, 3000], [64, 1, 17], 2, 4, 128, 32, bits)
    for _ in range(2):
        t.check(*t.run(workspace=big))
        o2, l2 = s.run(workspace=big, out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0))
        assert torch.equal(o2, out) and torch.equal(l2, lse)


@pytest.mark.parametrize("bits", [4, 16])
def test_many_sequences(bits):
    """More sequences than one warp takes at a time, empty ones among them."""
    rng = np.random.default_rng(8)
    n = 150
    contexts = [int(x) for x in rng.integers(0, 90, n)]
    nodes = [int(x) for x in rng.integers(0, 3, n)]
    contexts[40], nodes[40] = 2500, 2
    s = Setup(13, contexts, nodes, 2, 2, 64, 16, bits)
    s.check(*s.run(max_nodes=2))


@pytest.mark.parametrize("bits", [4, 16])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(bits):
    """A drafted token whose key, or whose value, holds NaN or infinity: its descendants see it, its siblings do not."""
    B, torch = _B(), _t()
    nodes = 6
    for context in (0, 5, 130):
        s = Setup(21, [context, 40], [nodes, 1], 1, 2, 128, 16, bits)
        masks = [1, 1 | 2, 1 | 4, 1 | 2 | 8, 16, 1 | 32]                       # token 1 is seen by tokens 1 and 3
        s.masks[0] = masks
        s.mask = torch.tensor(masks + [1, 0, 0], device="cuda")
        clean, clse = (x.clone() for x in s.run())
        s.check(clean, clse)
        pos = context + 1
        slot = s.dev["table"][0, pos // 16].long() * 16 + pos % 16
        for which in ("k", "v"):
            old = s.data.clone()
            k, v = (_dev(x[0][pos:pos + 1]) for x in (s.k, s.v))
            (k if which == "k" else v)[0, 0, 3] = float("nan")
            (k if which == "k" else v)[0, 0, 77] = float("inf")
            B.conqur_kv_append(s.cache, k, v, slot[None])
            out, lse = s.run(out=torch.full_like(clean, 7.0), lse=torch.full_like(clse, 7.0))
            s.data.copy_(old)
            hit = [1, 3]
            rest = [i for i in range(out.shape[0]) if i not in hit]
            assert torch.equal(out[rest], clean[rest]) and torch.equal(lse[rest], clse[rest])
            if which == "k" or bits == 4:
                assert torch.isnan(out[hit]).all()
            else:
                assert torch.isnan(out[hit][..., 3]).all() and torch.isinf(out[hit][..., 77]).all()
                keep = [e for e in range(128) if e not in (3, 77)]
                assert torch.equal(out[hit][..., keep], clean[hit][..., keep])


def test_bad_pages_contexts_and_starts_are_left_out_and_told_of():
    B, torch = _B(), _t()
    for bits in (4, 16):
        s = Setup(31, [100, 50, 70], [2, 3, 1], 2, 2, 64, 16, bits)
        good, glse = (x.clone() for x in s.run())
        assert B.conqur_kv_status() == 0
        fresh = dict(out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0))
        for value in (-1, 10 ** 6, 2 ** 31 - 1):
            old = s.dev["table"].clone()
            s.dev["table"][1, 1] = value                                       # positions 16 .. 31 of the second sequence
            out, lse = s.run(**fresh)
            assert B.conqur_kv_status() == -11 and B.conqur_kv_status() == 0
            assert torch.equal(out[:2], good[:2]) and torch.equal(out[5:], good[5:])
            for h in range(4):
                kh = h // 2
                seen = np.zeros((3, 53), bool)
                seen[:, :50] = True
                for i in range(3):
                    for j in range(3):
                        seen[i, 50 + j] = (s.masks[1][i] >> j) & 1
                seen[:, 16:32] = False
                want, _, mass, size = K.attend(s.q[2:5, h], s.k[1][:, kh], s.v[1][:, kh], seen, 64 ** -0.5)
                bound = (2.0 ** -8 + 2.0 ** -17 * size[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want)
                bound += _codes_bound(s.step[1][:, kh], s.k[1][:, kh], s.q[2:5, h], seen, 64 ** -0.5)
                assert (np.abs(out[2:5, h].float().cpu().numpy() - want) <= bound).all()
            s.dev["table"].copy_(old)
        # a table too narrow for a context, a negative context, more tokens than max_nodes, rows outside q
        wide = s.dev["table"]
        s.dev["table"] = wide[:, :4].contiguous()
        s.run(**fresh)
        assert B.conqur_kv_status() == -11
        s.dev["table"] = wide
        for name, at, value in (("contexts", 0, -5), ("starts", 3, 100), ("starts", 1, 6)):
            old = s.dev[name].clone()
            s.dev[name][at] = value
            s.run(out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0))
            s.dev[name].copy_(old)
            assert B.conqur_kv_status() == -11, name
        s.run(max_nodes=2, out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0))
        assert B.conqur_kv_status() == -11
        out, lse = s.run(**fresh)
        assert torch.equal(out, good) and torch.equal(lse, glse) and B.conqur_kv_status() == 0


def test_strided_queries_no_lse_streams_and_graphs():
    B, torch = _B(), _t()
    s = Setup(41, [300, 20], [3, 2], 2, 4, 128, 16, 4)
    good, glse = (x.clone() for x in s.run())
    fused = torch.zeros(s.rows, 20, 128, device="cuda").bfloat16()
    fused[:, 4:12] = s.dev["q"]
    s.dev["q"] = fused[:, 4:12]
    wide = torch.full((s.rows, 8, 136), 7.0, device="cuda").bfloat16()
    out, _ = s.run(out=wide[..., :128])
    assert torch.equal(out[:5], good[:5]) and (wide[..., 128:] == 7.0).all() and (wide[5:] == 7.0).all()
    # without lse, through the C call
    call = list(B._TREE_CALL.unpack(B._TREE_CALL.pack(B._TREE_CALL.size, 2, 4, 3, 128 ** -0.5, s.dev["table"].shape[1], s.rows, s.dev["q"].data_ptr(), 20 * 128, 128,
                                                      s.out.data_ptr(), 8 * 128, 128, 0, 0, s.dev["starts"].data_ptr(), s.dev["contexts"].data_ptr(),
                                                      s.dev["table"].data_ptr(), s.dev["table"].stride(0), s.mask.data_ptr(), 0, 0)))
    ws = B.attention_workspace(s.cache, 4, 3)
    call[-2:] = [ws.data_ptr(), ws.numel()]
    s.out.fill_(7.0)
    assert B.load().conqur_tree_attention(s.cache._ref, B._TREE_CALL.pack(*call), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(s.out, good)
    # another stream, with its own workspace, beside this one
    side, ws2 = torch.cuda.Stream(), B.attention_workspace(s.cache, 4, 3)
    outs = [torch.full_like(good, 7.0) for _ in range(2)]
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        s.run(out=outs[0], workspace=ws)
        with torch.cuda.stream(side):
            s.run(out=outs[1], lse=s.lse.clone(), workspace=ws2)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(outs[0], good) and torch.equal(outs[1], good)
    # captured once, replayed while the contexts grow: append and attention of a decoding step
    s = Setup(42, [0, 30], [1, 1], 2, 4, 128, 16, 4)
    width = 12
    table = torch.arange(2 * width, device="cuda", dtype=torch.int32).reshape(2, width)
    cache = B.KVCache(2 * width, 16, 2, 128, data=torch.full((2 * width, 2, K.block_bytes(16, 128, 4)), 0xFF, dtype=torch.uint8, device="cuda"))
    ws = B.attention_workspace(cache, 4, 1)
    ctx = torch.zeros(2, dtype=torch.int32, device="cuda")
    starts = torch.arange(3, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(2, h, 128, device="cuda").bfloat16() for h in (8, 2, 2))
    steps = [[torch.randn(2, h, 128, device="cuda").bfloat16() for h in (8, 2, 2)] for _ in range(40)]

    def step():
        pos = ctx.long()
        slots = table.gather(1, (pos // 16)[:, None])[:, 0].long() * 16 + pos % 16
        B.conqur_kv_append(cache, k, v, slots)
        out, lse = B.conqur_tree_attention(q, cache, starts, ctx, table, workspace=ws)
        ctx.add_(1)
        return out

    warm = step()
    ctx.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    ks, vs, sv = [], [], []
    for a, b, c in steps:
        q.copy_(a)
        k.copy_(b)
        v.copy_(c)
        graph.replay()
        sv.append(K.quantise(c.float().cpu().numpy().astype(np.float64))[2][..., 0])
        ks.append(K.values(b.float().cpu().numpy().astype(np.float64), 4))
        vs.append(K.values(c.float().cpu().numpy().astype(np.float64), 4))
        if len(ks) in (1, 16, 17, 33, 40):
            for i in range(2):
                for h in range(8):
                    kk, vv = np.array([x[i, h // 4] for x in ks]), np.array([x[i, h // 4] for x in vs])
                    qq = a[i, h].float().cpu().numpy()[None]
                    want, _, mass, size = K.attend(qq, kk, vv, np.ones((1, len(ks)), bool), 128 ** -0.5)
                    bound = (2.0 ** -8 + 2.0 ** -17 * size[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want)
                    bound += _codes_bound(np.array([x[i, h // 4] for x in sv]), kk, qq, np.ones((1, len(ks)), bool), 128 ** -0.5)
                    assert (np.abs(out[i, h].float().cpu().numpy() - want) <= bound).all()
    assert B.conqur_kv_status() == 0 and warm.shape == out.shape


@pytest.mark.parametrize("bits", [4, 16])
def test_more_rows_long_split_many_sequences_and_rising_scores(bits):
    """More than 16 rows a key head: an item over many CTAs, the same bits again through one workspace; more sequences than a warp takes at a time, some
    empty; scores whose maximum rises along the positions."""
    B, torch = _B(), _t()
    s = Setup(71, [20000], [20], 2, 4, 128, 64, bits)
    ws = B.attention_workspace(s.cache, 4, 20)
    out, lse = s.run(workspace=ws)
    s.check(out, lse)
    for _ in range(3):
        o2, l2 = s.run(workspace=ws, out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0))
        assert torch.equal(o2, out) and torch.equal(l2, lse)
    rng = np.random.default_rng(72)
    contexts, nodes = [int(x) for x in rng.integers(0, 200, 75)], [int(x) for x in rng.integers(0, 5, 75)]
    contexts[50], nodes[50] = 3000, 4
    m = Setup(73, contexts, nodes, 2, 6, 64, 16, bits)
    m.check(*m.run(max_nodes=4))
    u = Setup(74, [700, 130, 64], [9, 20, 3], 1, 4, 128, 32, bits, sharp=12.0)
    u.check(*u.run())
    assert B.conqur_kv_status() == 0


@pytest.mark.parametrize("bits", [4, 16])
def test_more_rows_values_that_are_not_finite_bad_pages_and_odd_queries(bits):
    """More than 16 rows a key head: NaN and infinity in a drafted token's key or value, in a context token's value, in one query; pages that are not there."""
    B, torch = _B(), _t()
    nodes, group = 6, 8
    for context in (0, 5, 130):
        s = Setup(81, [context, 40], [nodes, 1], 1, group, 128, 16, bits)
        masks = [1, 1 | 2, 1 | 4, 1 | 2 | 8, 16, 1 | 32]                       # token 1 is seen by tokens 1 and 3
        s.masks[0] = masks
        s.mask = torch.tensor(masks + [1, 0, 0], device="cuda")
        clean, clse = (x.clone() for x in s.run())
        s.check(clean, clse)
        fresh = lambda: dict(out=torch.full_like(clean, 7.0), lse=torch.full_like(clse, 7.0))
        for pos, hit in ((context + 1, [1, 3]), (context // 2, list(range(nodes)))):
            if pos == context and context == 0:
                continue
            slot = s.dev["table"][0, pos // 16].long() * 16 + pos % 16
            for which in ("k", "v"):
                old = s.data.clone()
                k, v = (_dev(x[0][pos:pos + 1]) for x in (s.k, s.v))
                (k if which == "k" else v)[0, 0, 3] = float("nan")
                (k if which == "k" else v)[0, 0, 77] = float("inf")
                B.conqur_kv_append(s.cache, k, v, slot[None])
                out, lse = s.run(**fresh())
                s.data.copy_(old)
                rest = [i for i in range(out.shape[0]) if i not in hit]
                assert torch.equal(out[rest], clean[rest]) and torch.equal(lse[rest], clse[rest])
                if which == "k" or bits == 4:
                    assert torch.isnan(out[hit]).all()
                else:
                    assert torch.isnan(out[hit][..., 3]).all() and torch.isinf(out[hit][..., 77]).all()
        # one query row
        q = s.dev["q"].clone()
        s.dev["q"][2, 5, 60] = float("nan")
        out, lse = s.run(**fresh())
        s.dev["q"] = q
        assert torch.isnan(out[2, 5]).all() and torch.isnan(lse[2, 5])
        out[2, 5], lse[2, 5] = clean[2, 5], clse[2, 5]
        assert torch.equal(out, clean) and torch.equal(lse, clse)
    assert B.conqur_kv_status() == 0
    s.dev["table"][0, 3] = 10 ** 6                                             # positions 48 .. 63 of the first sequence
    out, lse = s.run(**fresh())
    assert B.conqur_kv_status() == -11 and torch.equal(out[nodes:], clean[nodes:])
    seen = np.zeros((nodes, context + nodes), bool)
    seen[:, :context] = True
    for i in range(nodes):
        for j in range(nodes):
            seen[i, context + j] = (masks[i] >> j) & 1
    seen[:, 48:64] = False
    for h in range(group):
        want, _, mass, size = K.attend(s.q[:nodes, h], s.k[0][:, 0], s.v[0][:, 0], seen, 128 ** -0.5)
        bound = (2.0 ** -8 + 2.0 ** -17 * size[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want)
        bound += _codes_bound(s.step[0][:, 0], s.k[0][:, 0], s.q[:nodes, h], seen, 128 ** -0.5)
        assert (np.abs(out[:nodes, h].float().cpu().numpy() - want) <= bound).all()


def test_more_rows_on_two_streams_and_in_a_graph():
    """More than 16 rows a key head: two calls at once with workspaces of their own, and a captured call replayed with other lengths."""
    B, torch = _B(), _t()
    s = Setup(91, [900, 2500, 64], [8, 5, 8], 2, 4, 128, 32, 4)
    good, glse = (x.clone() for x in s.run())
    s.check(good, glse)
    ws = [B.attention_workspace(s.cache, 4, 8) for _ in range(2)]
    outs = [torch.full_like(good, 7.0) for _ in range(2)]
    lses = [torch.full_like(glse, 7.0) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        s.run(out=outs[0], lse=lses[0], workspace=ws[0])
        with torch.cuda.stream(side):
            s.run(out=outs[1], lse=lses[1], workspace=ws[1])
    torch.cuda.current_stream().wait_stream(side)
    for o, l in zip(outs, lses):
        assert torch.equal(o, good) and torch.equal(l, glse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(out=outs[0], lse=lses[0], workspace=ws[0])
    old = s.contexts
    for cut in (0, 1, 63):
        s.contexts = [c - cut for c in old]
        s.dev["contexts"].copy_(torch.tensor(s.contexts, dtype=torch.int32))
        # the drafted tokens are then those that lie behind the shorter context
        outs[0].fill_(7.0)
        lses[0].fill_(7.0)
        graph.replay()
        keep = [(k, v) for k, v in zip(s.k, s.v)], s.step
        s.k, s.v = [k[: c + n] for k, c, n in zip(s.k, s.contexts, s.nodes)], [v[: c + n] for v, c, n in zip(s.v, s.contexts, s.nodes)]
        s.step = [x[: c + n] for x, c, n in zip(s.step, s.contexts, s.nodes)]
        s.check(outs[0], lses[0])
        s.k, s.v, s.step = [x[0] for x in keep[0]], [x[1] for x in keep[0]], keep[1]
    assert B.conqur_kv_status() == 0


def test_cache_past_4_gigabytes():
    """Pages whose byte offset needs more than 32 bits, and slots past 2^22."""
    B, torch = _B(), _t()
    page, heads, d = 64, 8, 128
    pages = (2 ** 32) // (heads * K.block_bytes(page, d, 4)) + 40
    cache = B.KVCache(pages, page, heads, d)
    s = Setup(51, [150], [2], heads, 2, d, page, 4)
    used = int(-(-152 // page))
    far = torch.arange(pages - used, pages, device="cuda")
    near = s.dev["table"][0, :used].long()
    cache.data[far] = s.data[near]
    good, glse = s.run()
    out = torch.full_like(good, 7.0)
    lse = torch.full_like(glse, 7.0)
    B.conqur_tree_attention(s.dev["q"], cache, s.dev["starts"], s.dev["contexts"], far.int()[None], s.mask, max_nodes=2, out=out, lse=lse)
    assert torch.equal(out, good) and torch.equal(lse, glse)
    k = torch.randn(3, heads, d, device="cuda").bfloat16()
    slots = torch.tensor([pages * page - 1, pages * page - 7, 5], device="cuda")
    B.conqur_kv_append(cache, k, -k, slots)
    kr, vr = B.conqur_kv_read(cache, slots, torch.float32)
    ref = K.values(k.float().cpu().numpy().astype(np.float64), 4)
    assert np.array_equal(kr.cpu().numpy().astype(np.float64), ref) and B.conqur_kv_status() == 0


def test_rotated_heads_through_the_cache_to_attention():
    """The operators as they are used: normed, rotated and Hadamard-transformed heads, keys into the 4-bit cache, attention of a tree."""
    from oracle import heads_oracle as H
    B, torch = _B(), _t()
    hq, hk, d, page, ctx, nodes = 8, 2, 128, 16, 90, 5
    r = np.random.default_rng(61)
    rope = B.Rope(d, theta=500000.0, layout="half", scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192)
    n = ctx + nodes
    qkv = _dev(K.bf16(r.standard_normal((n, hq + 2 * hk, d))))
    wq, wk = (_dev(K.bf16(1 + 0.2 * r.standard_normal(d))) for _ in range(2))
    pos = torch.arange(n, device="cuda") + 30000
    q, k = B.conqur_norm_rope_heads(qkv[:, :hq], qkv[:, hq:hq + hk], wq, wk, pos, rope, 1e-6, hadamard=True)
    cache = B.KVCache(8, page, hk, d)
    table = torch.tensor([[5, 0, 7, 2, 3, 6, 1]], dtype=torch.int32, device="cuda")[:, : -(-n // page)].contiguous()
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page] * page + at % page
    B.conqur_kv_append(cache, k, qkv[:, hq + hk:], slots)
    masks = [1, 3, 5, 11, 17]
    out, _ = B.conqur_tree_attention(q[ctx:].contiguous(), cache, torch.tensor([0, nodes], dtype=torch.int32, device="cuda"),
                                     torch.tensor([ctx], dtype=torch.int32, device="cuda"), table, torch.tensor(masks, device="cuda"), max_nodes=nodes)
    # the same from the formulas; stored heads carry one bf16 rounding, keys and values the cache's codes
    x = qkv.float().cpu().numpy().astype(np.float64)
    f, amp = H.frequencies(d, theta=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192)
    w = [t.float().cpu().numpy().astype(np.float64) for t in (wq, wk)]
    q64 = H.norm_rotate(x[:, :hq], w[0], 1e-6, pos.cpu().numpy(), f, amp, "half", True)
    assert np.abs(q.float().cpu().numpy() - q64).max() <= 2.0 ** -8 * np.abs(q64).max()
    kv = K.values(k.float().cpu().numpy().astype(np.float64), 4), K.values(x[:, hq + hk:], 4)
    seen = np.zeros((nodes, n), bool)
    seen[:, :ctx] = True
    for i in range(nodes):
        for j in range(nodes):
            seen[i, ctx + j] = (masks[i] >> j) & 1
    qs = q[ctx:].float().cpu().numpy()
    for h in range(hq):
        want, _, mass, size = K.attend(qs[:, h], kv[0][:, h // 4], kv[1][:, h // 4], seen, d ** -0.5)
        bound = (2.0 ** -8 + 2.0 ** -17 * size[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want)
        bound += _codes_bound(K.quantise(x[:, hq + hk:])[2][:, h // 4, 0], kv[0][:, h // 4], qs[:, h], seen, d ** -0.5)
        assert (np.abs(out[:, h].float().cpu().numpy() - want) <= bound).all()
    assert B.conqur_kv_status() == 0
