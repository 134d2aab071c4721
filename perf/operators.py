"""Operators between a model's q/k/v projections and its attention output, as cases that can be timed and compared with 64-bit
arithmetic: the plain forms (elementary torch operations) and the framework's calls on the same inputs.

Kinds of case (``kind``):

  rope      position rotation of query and key heads (half or interleaved pairs, the whole head or its first part, frequencies
            scaled for long contexts), optionally followed by the online Hadamard rotation R_3; ``inverse`` is its backward pass
  norm      RMS norm of every query and key head, then the rotation, in one pass; ``grad`` is the backward pass (gradients of the
            heads and of the two shared weights)
  append    keys and values written into the paged cache (4-bit zero-point codes or bf16) and read back as values
  attend    attention of drafted tokens (a tree per sequence; a tree of one token is ordinary decoding) over that cache

Sizes are those of 7B/8B- and 70B-class models with heads of 128 (32 or 64 query heads, 8 or 32 key heads) or generic; values
follow the recipe of ``paper_2605_10793_b200/inputs.py`` (Student-t(3) entries, outlier channels, a scale per token).

Cache layout (pages of ``page`` tokens; one contiguous block per page and key head, page after page, head after head):

  4 bits   key codes page x D/2 bytes, value codes page x D/2 bytes, key records page x 4 bytes, value records page x 4 bytes.
           Nibble i (i = 0 lowest) of the 32-bit word w of a token's row holds dimension 8 w + (0, 2, 4, 6, 1, 3, 5, 7)[i]; a record is
           the step as bf16 (low half) and the zero-point code (high half); value = (code - zero-point) * step
  16 bits  keys, then values, each D/64 planes of page x 64 bf16; 16-byte piece j of token t's 128-byte row lies at piece j ^ (t & 7)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}

# Frequencies: theta^(-2i/r), and how a context longer than the trained one rescales them.
_SCALING = {
    "none": dict(theta=10000.0),
    "linear": dict(theta=10000.0, factor=8.0),
    "ntk": dict(theta=10000.0, factor=4.0),
    "bands": dict(theta=500000.0, factor=8.0, low=1.0, high=4.0, original=8192),
    "ramp": dict(theta=10000.0, factor=16.0, low=1.0, high=32.0, original=4096),
}


def _case(kind, name=None, **kw):
    base = {
        "rope": dict(n=4096, hq=32, hk=8, d=128, rot=128, layout="half", scaling="none", dtype="bf16", r3=False, inverse=False,
                     far=4096, spread=False),
        "norm": dict(n=4096, hq=32, hk=8, d=128, rot=128, layout="half", scaling="none", dtype="bf16", r3=False, grad=False,
                     far=4096, spread=False),
        "append": dict(n=4096, hk=8, d=128, page=64, bits=4, clip=1.0, pages=512, scattered=False),
        "attend": dict(b=8, context=4096, ragged=True, nodes=1, chain=False, hk=8, group=4, d=128, page=64, bits=4),
    }[kind]
    out = dict(kind=kind, **base)
    out.update(kw)
    if name:
        out["name"] = name
    return out


def listed():
    return [
        # one decoding step of a batch of long conversations, 8B-class heads, wavelength-band frequencies: latency
        _case("rope", "rope_decode_far", n=33, scaling="bands", far=120000, spread=True),
        # prompts of an 8B-class model on their way into a 4-bit cache: rotation and R_3 in one pass
        _case("rope", "rope_prompt_r3", n=16384, scaling="bands", r3=True, far=8192),
        # backward pass of a partial, interleaved rotation in fp32, ragged
        _case("rope", "rope_partial_grad_f32", n=4001, hq=16, hk=16, d=96, rot=32, layout="interleaved", dtype="f32", inverse=True),
        # decoding with normed heads and R_3
        _case("norm", "norm_decode_r3", n=64, r3=True, far=32768, spread=True),
        # a training batch, forward ...
        _case("norm", "norm_prompt_ramp", n=8192, scaling="ramp", far=16384),
        # ... and backward
        _case("norm", "norm_prompt_grad", n=8192, grad=True),
        # one decoding step of a batch: a row per sequence into scattered pages, some rows padding
        _case("append", "append_decode_kv4", n=97, pages=1024, scattered=True),
        # prompts into a 4-bit cache
        _case("append", "append_prompt_kv4", n=32768, pages=600),
        # a batch of short sequences, seven drafted tokens each, heads of 64, bf16 cache: latency
        _case("attend", "attend_small_tree_kv16", b=3, context=700, nodes=7, hk=4, group=2, d=64, page=16, bits=16),
        # decoding with a 4-bit cache, ragged contexts
        _case("attend", "attend_decode_kv4", b=64, context=8192),
        # one long conversation, bf16 cache
        _case("attend", "attend_long_kv16", b=1, context=131071, ragged=False, bits=16),
        # a tree of drafted tokens over a 4-bit cache
        _case("attend", "attend_tree_kv4", b=16, context=6000, nodes=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "norm", "norm", "append", "attend", "attend", "attend"])
    if kind in ("rope", "norm"):
        hq, hk = rng.choice([(32, 8), (32, 32), (64, 8), (28, 4), (16, 16), (8, 1), (5, 5), (3, 2)])
        d = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        kw = dict(hq=hq, hk=hk, d=d, rot=rng.choice([d, d, d, d // 2, d // 4 // 2 * 2]), layout=rng.choice(["half", "half", "interleaved"]),
                  scaling=rng.choice(sorted(_SCALING)), dtype=dtype, r3=d in (64, 128, 256) and rng.random() < 0.5,
                  far=_log_int(rng, 64, 1 << 20), spread=rng.random() < 0.4)
        kw["inverse" if kind == "rope" else "grad"] = rng.random() < 0.4
        return _case(kind, n=_log_int(rng, 1, 16384 * 40 * 128 // ((hq + hk) * d * (2 if dtype == "f32" else 1) * (2 if kw.get("grad") else 1))), **kw)
    if kind == "append":
        hk, d = rng.choice([(8, 128), (32, 128), (4, 64), (1, 128), (5, 64)])
        page = rng.choice([16, 32, 64])
        n = _log_int(rng, 1, 32768 * 8 * 128 // (hk * d))
        return _case(kind, n=n, hk=hk, d=d, page=page, bits=rng.choice([4, 4, 16]), clip=rng.choice([1.0, 1.0, 0.9]),
                     pages=n // page + 2 + rng.randrange(64), scattered=rng.random() < 0.5)
    hk, group = rng.choice([(8, 4), (8, 8), (32, 1), (4, 7), (1, 16), (2, 5), (4, 2)])
    d, bits = rng.choice([64, 128, 128]), rng.choice([4, 4, 16])
    nodes = rng.choice([1, 1, 1, rng.randrange(2, 17), rng.randrange(17, 65)])
    b = _log_int(rng, 1, 128)
    # bytes of the largest listed cache, and operations of the largest listed tree
    most = min(540e6 / (b * hk * d * (4 if bits == 16 else 1)), 16 * 8 * 128 * 6000 * 1.2 * 128 / (b * hk * group * nodes * d), 131072)
    return _case(kind, b=b, context=_log_int(rng, 1, max(2, int(most))), ragged=rng.random() < 0.7, nodes=nodes, chain=rng.random() < 0.3,
                 hk=hk, group=group, d=d, page=rng.choice([16, 32, 64]), bits=bits)


# ---- inputs -------------------------------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1013 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _heads(g, n, h, d, dtype):
    """n x h x d head rows: Student-t(3) entries, two outlier channels a head, a scale per token; in the storage type."""
    out = torch.empty(n, h, d, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // (h * d))
    loud = torch.ones(h, d, device="cuda").scatter_(1, torch.rand(h, d, generator=g, device="cuda").argsort(dim=1)[:, :2], 8.0)
    for a in range(0, n, step):
        m = min(step, n - a)
        c = (_randn(g, m, h, d).square_() + _randn(g, m, h, d).square_() + _randn(g, m, h, d).square_()) * (1.0 / 3.0)
        x = _randn(g, m, h, d).mul_(c.rsqrt_()).mul_(loud).mul_(torch.exp(0.5 * _randn(g, m, 1, 1)))
        out[a:a + m] = x.to(dtype)
    return out


def _frequencies(case):
    """(r/2 angular frequencies in 64 bits, amplitude) of the case's position rotation."""
    s, r = _SCALING[case["scaling"]], case["rot"]
    i = torch.arange(r // 2, dtype=torch.float64)
    theta, factor = s["theta"], s.get("factor", 1.0)
    if case["scaling"] == "ntk" and r > 2:
        theta = theta * factor ** (r / (r - 2))
    f = theta ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "bands":
        # turns made over the trained context: many keep their frequency, few are stretched, a linear passage between
        smooth = ((s["original"] * f / (2 * math.pi) - s["low"]) / (s["high"] - s["low"])).clamp(0, 1)
        return f * (smooth + (1 - smooth) / factor), 1.0
    if case["scaling"] == "ramp":
        where = [r * math.log(s["original"] / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (s["high"], s["low"])]
        a, b = max(math.floor(where[0]), 0), min(math.ceil(where[1]), r - 1)
        ramp = ((i - a) / max(b - a, 0.001)).clamp(0, 1)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _hadamard_matrix(d):
    """The symmetric orthogonal Sylvester matrix: entry (i, j) is (-1)^(bits that i and j share) / sqrt(d)."""
    h = torch.ones(1, 1, device="cuda")
    while h.shape[0] < d:
        h = torch.cat((torch.cat((h, h), dim=1), torch.cat((h, -h), dim=1)))
    return h / math.sqrt(d)


def _positions(g, case):
    n, far = case["n"], case["far"]
    if case["spread"]:
        return torch.randint(0, far, (n,), generator=g, device="cuda")
    length = min(n, far)                                    # prompts of one length, one after another, the last one cut off
    return torch.arange(n, device="cuda") % length + (far - length)


def _make_cache(g, pages, case):
    """A cache as it lies in memory before anything is written: its bytes say nothing (here they would read as NaN)."""
    per = case["page"] * (case["d"] + 8) if case["bits"] == 4 else case["page"] * case["d"] * 4
    return torch.full((pages, case["hk"], per), 0xFF, dtype=torch.uint8, device="cuda")


def _fill(g, cache, table, lengths, case):
    """Keys and values of every sequence's first ``lengths`` positions, written page by page."""
    p, hk, d = case["page"], case["hk"], case["d"]
    used = [table[b, : -(-int(n) // p)] for b, n in enumerate(lengths)]
    owner = torch.cat([torch.full((len(u),), b, device="cuda") for b, u in enumerate(used)])
    first = torch.cat([torch.arange(len(u), device="cuda") * p for u in used])
    used = torch.cat(used).long()
    have = torch.as_tensor(lengths, device="cuda")[owner] - first
    step = max(1, (1 << 26) // (p * hk * d))
    for a in range(0, len(used), step):
        pg = used[a:a + step]
        k, v = (_randn(g, len(pg), p, hk, d) for _ in range(2))
        k[..., : d // 16] *= 3.0
        slots = pg[:, None] * p + torch.arange(p, device="cuda")
        slots = torch.where(torch.arange(p, device="cuda") < have[a:a + step, None], slots, -1).reshape(-1)
        _plain_append(cache, k.reshape(-1, hk, d).bfloat16(), v.reshape(-1, hk, d).bfloat16(), slots, case, wide=torch.float32)


def _nodes(case):
    """Drafted tokens of each sequence."""
    t = case["nodes"]
    return [t - (5 * i) % (t - t // 2) if case["ragged"] and t > 1 else t for i in range(case["b"])]


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("rope", "norm"):
        n, hq, hk, d, dt = case["n"], case["hq"], case["hk"], case["d"], _DT[case["dtype"]]
        fused = _heads(g, n, hq + 2 * hk, d, dt)            # rows of a fused q/k/v projection
        s["q"], s["k"] = fused[:, :hq], fused[:, hq:hq + hk]
        s["pos"] = _positions(g, case)
        s["freq"], s["amp"] = _frequencies(case)
        s["freq"] = s["freq"].cuda()
        if case["r3"]:
            s["r3"] = _hadamard_matrix(d)
        if kind == "norm":
            s["eps"] = 1e-6
            s["wq"], s["wk"] = ((1.0 + 0.2 * _randn(g, d)).to(dt) for _ in range(2))
            if case["grad"]:
                s["gq"], s["gk"] = (_randn(g, n, h, d).to(dt) for h in (hq, hk))
    elif kind == "append":
        n, hk, d, p = case["n"], case["hk"], case["d"], case["page"]
        fused = _heads(g, n, 2 * hk, d, torch.bfloat16)
        s["k"], s["v"] = fused[:, :hk], fused[:, hk:]
        s["cache"] = _make_cache(g, case["pages"], case)
        total = case["pages"] * p
        s["slots"] = torch.randperm(total, generator=g, device="cuda")[:n] if case["scattered"] else torch.arange(n, device="cuda") + (total - n) // 2
        pad = torch.rand(n, generator=g, device="cuda") < (0.1 if n > 1 else 0.0)
        s["slots"][pad] = -1
    else:
        b, t, hk, d, p = case["b"], case["nodes"], case["hk"], case["d"], case["page"]
        r = np.random.default_rng([int(seed) & 0x7FFFFFFF, 31])
        context = r.integers(case["context"] // 2, case["context"] + 1, b) if case["ragged"] else np.full(b, case["context"])
        nodes = np.array(_nodes(case))
        starts = np.concatenate([[0], np.cumsum(nodes)])
        lengths = context + nodes
        width = int(-(-lengths.max() // p))
        need = -(-lengths // p)
        pages = int(need.sum()) + 3
        order = torch.randperm(pages, generator=g, device="cuda").int()
        table = torch.zeros(b, width, dtype=torch.int32, device="cuda")
        at = np.concatenate([[0], np.cumsum(need)])
        for i in range(b):
            table[i, : need[i]] = order[at[i]:at[i + 1]]
        # a node sees itself and its ancestors: bit j of the mask of node i
        mask = np.zeros(starts[-1], dtype=np.uint64)
        for i in range(b):
            for j in range(nodes[i]):
                parent = j - 1 if case["chain"] else int(r.integers(max(0, j - 4), j)) if j else -1
                up = mask[starts[i] + parent] if parent >= 0 else np.uint64(0)
                mask[starts[i] + j] = up | np.uint64(1 << j)
        s["mask"] = torch.from_numpy(mask.view(np.int64)).cuda()
        s["starts"] = torch.from_numpy(starts.astype(np.int32)).cuda()
        s["contexts"] = torch.from_numpy(context.astype(np.int32)).cuda()
        s["table"] = table
        s["cache"] = _make_cache(g, pages, case)
        _fill(g, s["cache"], table, lengths, case)
        s["q"] = 1.5 * _randn(g, int(starts[-1]), hk * case["group"], d)
        s["q"] = s["q"].bfloat16()
        s["longest"] = int(lengths.max())
        s["scale"] = 1.0 / math.sqrt(d)
    return s


# ---- the framework's calls ----------------------------------------------------------------------------------------



B = None


def _own(s):
    global B
    if B is None:
        from paper_2605_10793_b200 import binding as B
    case = s["case"]
    kind = case["kind"]
    if kind in ("rope", "norm"):
        if "rope" not in s:                                 # a program makes its frequency table once
            f = _SCALING[case["scaling"]]
            s["rope"] = B.Rope(case["rot"], theta=f["theta"], layout=case["layout"], scaling=case["scaling"], factor=f.get("factor", 1.0),
                               low=f.get("low", 0.0), high=f.get("high", 0.0), original=f.get("original", 0))
        if kind == "rope":
            return B.conqur_rope_heads(s["q"], s["k"], s["pos"], s["rope"], hadamard=case["r3"], inverse=case["inverse"])
        if case["grad"]:
            return B.conqur_norm_rope_heads_backward(s["gq"], s["gk"], s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["rope"], s["eps"],
                                                     hadamard=case["r3"])
        return B.conqur_norm_rope_heads(s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["rope"], s["eps"], hadamard=case["r3"])
    if "handle" not in s:
        s["handle"] = B.KVCache(s["cache"].shape[0], case["page"], case["hk"], case["d"], bits=case["bits"],
                                clip_ratio=case.get("clip", 1.0), data=s["cache"])
    if kind == "append":
        B.conqur_kv_append(s["handle"], s["k"], s["v"], s["slots"])
        return B.conqur_kv_read(s["handle"], s["slots"])
    if "space" not in s:
        s["space"] = B.attention_workspace(s["handle"], case["group"], case["nodes"])
    return B.conqur_tree_attention(s["q"], s["handle"], s["starts"], s["contexts"], s["table"], s["mask"], max_nodes=case["nodes"],
                                   scale=s["scale"], workspace=s["space"])


# ---- the plain forms ----------------------------------------------------------------------------------------------


def _turn(x, s, sign):
    """x (n, heads, d) in fp32 with its first ``rot`` dimensions rotated by sign * position * frequency."""
    case = s["case"]
    r = case["rot"]
    angle = s["pos"].double()[:, None] * s["freq"]
    c = (s["amp"] * torch.cos(angle)).float()[:, None, :]
    t = (s["amp"] * sign * torch.sin(angle)).float()[:, None, :]
    part, rest = x[..., :r], x[..., r:]
    if case["layout"] == "half":
        a, b = part[..., : r // 2], part[..., r // 2:]
        return torch.cat((a * c - b * t, a * t + b * c, rest), dim=-1)
    a, b = part[..., 0::2], part[..., 1::2]
    return torch.cat((torch.stack((a * c - b * t, a * t + b * c), dim=-1).flatten(-2), rest), dim=-1)


def _plain_heads(s):
    case = s["case"]
    out = []
    for name in ("q", "k"):
        x = s[name].float()
        if case["kind"] == "norm":
            x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + s["eps"]) * s["w" + name].float()
        if case.get("inverse"):
            x = _turn(x @ s["r3"] if case["r3"] else x, s, -1.0)
        else:
            x = _turn(x, s, 1.0)
            x = x @ s["r3"] if case["r3"] else x
        out.append(x.to(s[name].dtype))
    return tuple(out)


def _plain_norm_grad(s):
    case = s["case"]
    dx, dw = [], []
    for name in ("q", "k"):
        x, w, g = s[name].float(), s["w" + name].float(), s["g" + name].float()
        g = _turn(g @ s["r3"] if case["r3"] else g, s, -1.0)
        rstd = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + s["eps"])
        unit = x * rstd
        dw.append((g * unit).sum(dim=(0, 1)))
        g = g * w
        dx.append((rstd * (g - unit * (g * unit).mean(dim=-1, keepdim=True))).to(s[name].dtype))
    return dx[0], dx[1], dw[0], dw[1]


_NIBBLE = (0, 2, 4, 6, 1, 3, 5, 7)                          # dimension of each nibble within a 32-bit word


def _quantise(y, clip, wide):
    """(codes, zero-point codes, steps as bf16) of rows: the range is widened to hold 0, so the zero-point is a code too."""
    y = y.to(wide)
    clip = float(np.float32(clip))
    lo, hi = clip * y.amin(dim=-1, keepdim=True).clamp(max=0), clip * y.amax(dim=-1, keepdim=True).clamp(min=0)
    step = ((hi - lo) / 15).float().bfloat16()
    step = torch.where(step < 2.0 ** -100, torch.zeros_like(step), step)
    by = torch.where(step > 0, step, torch.ones_like(step)).to(wide)
    zero = torch.where(step > 0, -torch.round(lo / by), torch.zeros_like(lo)).clamp(0, 15)
    codes = torch.where(step > 0, (torch.round(y / by) + zero).clamp(0, 15), torch.zeros_like(y))
    return codes, zero, step


def _planes(cache, case):
    """Views of the cache's parts: (key codes, value codes, key records, value records) or (keys, values)."""
    p, d = case["page"], case["d"]
    if case["bits"] == 4:
        a = p * d // 2
        return (cache[..., :a].unflatten(-1, (p, d // 2)), cache[..., a:2 * a].unflatten(-1, (p, d // 2)),
                cache[..., 2 * a:2 * a + 4 * p].unflatten(-1, (p, 4)), cache[..., 2 * a + 4 * p:].unflatten(-1, (p, 4)))
    a = p * d * 2
    return tuple(c.unflatten(-1, (d // 64, p, 8, 16)) for c in (cache[..., :a], cache[..., a:]))


def _swizzle(case):
    """Piece of a token's row -> place of that piece, for every token of a page."""
    t = torch.arange(case["page"], device="cuda")
    return torch.arange(8, device="cuda")[None, :] ^ (t[:, None] & 7)


def _plain_append(cache, k, v, slots, case, wide=torch.float64):
    """Rows k, v (n, heads, d) in bf16 into their slots; a negative slot is a row that is not stored."""
    p, d = case["page"], case["d"]
    keep = slots >= 0
    slots = slots[keep]
    pg, t = slots // p, slots % p
    parts = _planes(cache, case)
    for i, y in enumerate((k[keep], v[keep])):
        if case["bits"] == 4:
            codes, zero, step = _quantise(y, case.get("clip", 1.0), wide)
            nib = codes.to(torch.uint8).unflatten(-1, (d // 8, 8))[..., list(_NIBBLE)]
            parts[i][pg, :, t] = (nib[..., 0::2] | (nib[..., 1::2] << 4)).flatten(-2)
            parts[2 + i][pg, :, t] = torch.cat((step.view(torch.int16), zero.to(torch.int16)), dim=-1).view(torch.uint8)
        else:
            pieces = y.contiguous().view(torch.uint8).unflatten(-1, (d // 64, 8, 16))     # n, heads, planes, 8, 16
            to = _swizzle(case)[t]
            pieces = pieces.gather(3, to[:, None, None, :, None].expand_as(pieces))       # x ^ c is its own inverse
            parts[i][pg, :, :, t] = pieces


def _token_values(parts, i, rows, t, case):
    """Keys (i = 0) or values (i = 1) in fp32 of the tokens that ``rows`` indexes in each plane; ``t``: their places in their pages."""
    d = case["d"]
    if case["bits"] == 4:
        c = rows(parts[i])
        nib = torch.stack((c & 15, c >> 4), dim=-1).flatten(-2).unflatten(-1, (d // 8, 8))
        back = [_NIBBLE.index(e) for e in range(8)]
        rec = rows(parts[2 + i]).contiguous()
        step, zero = rec.view(torch.bfloat16)[..., 0:1].float(), rec.view(torch.int16)[..., 1:2].float()
        return (nib[..., back].flatten(-2).float() - zero) * step
    c = rows(parts[i].movedim(-4, -3))                      # ..., planes, 8, 16
    place = (torch.arange(8, device="cuda") ^ (t[..., None] & 7))[..., None, :, None]
    return c.gather(-2, place.expand_as(c)).view(torch.bfloat16).float().flatten(-3)


def _values(blocks, case):
    """Keys and values (..., page, d) in fp32 of cache blocks (..., bytes)."""
    parts = _planes(blocks, case)
    return [_token_values(parts, i, lambda x: x, torch.arange(case["page"], device="cuda"), case) for i in range(2)]


def _plain_read(cache, slots, case):
    p, at = case["page"], slots.clamp(min=0)
    parts = _planes(cache, case)
    out = []
    for i in range(2):
        x = _token_values(parts, i, lambda c: c[at // p, :, at % p], (at % p)[:, None], case)        # n, heads, d
        out.append(torch.where((slots >= 0)[:, None, None], x, torch.zeros_like(x)).bfloat16())
    return tuple(out)


def _plain_attend(s):
    case = s["case"]
    b, t, hk, grp, d, p = (case[x] for x in ("b", "nodes", "hk", "group", "d", "page"))
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in _values(s["cache"][s["table"].long()], case))   # b, heads, positions, d
    n = s["longest"]
    k, v = k[:, :, :n], v[:, :, :n]
    starts, context = s["starts"].long(), s["contexts"].long()
    count = starts[1:] - starts[:-1]
    node = torch.arange(t, device="cuda")
    row = (starts[:-1, None] + node).clamp(max=s["q"].shape[0] - 1)                                   # b, t
    q = s["q"].float()[row].unflatten(2, (hk, grp)).permute(0, 2, 1, 3, 4).flatten(2, 3)             # b, heads, t * group, d
    j = torch.arange(n, device="cuda") - context[:, None]                                            # b, positions
    bit = (s["mask"][row][:, :, None] >> j.clamp(0, 63)[:, None, :]) & 1
    see = (j < 0)[:, None, :] | ((j >= 0) & (j < count[:, None]))[:, None, :] & (bit == 1)            # b, t, positions
    see = see & (node < count[:, None])[:, :, None]
    v = torch.where((j < count[:, None])[:, None, :, None], v, torch.zeros_like(v))
    see = see[:, None, :, None, :].expand(b, 1, t, grp, n).flatten(2, 3)
    x = torch.where(see, (q @ k.transpose(2, 3)) * s["scale"], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    e = torch.where(see, torch.exp(x - top), torch.zeros_like(x))
    total = e.sum(dim=-1, keepdim=True)
    o = torch.where(total > 0, (e @ v) / total, torch.zeros(1, device="cuda"))
    lse = torch.where(total > 0, top + torch.log(total), float("-inf"))
    real = (node < count[:, None])                                                                   # b, t
    o = o.unflatten(2, (t, grp)).transpose(1, 2).flatten(2, 3)[real]
    lse = lse.unflatten(2, (t, grp)).transpose(1, 2)[..., 0].flatten(2, 3)[real]
    return o.bfloat16(), lse


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    if case["kind"] == "append":
        _plain_append(s["cache"], s["k"], s["v"], s["slots"], case)
        return _plain_read(s["cache"], s["slots"], case)
    if case["kind"] == "attend":
        return _plain_attend(s)
    return _plain_norm_grad(s) if case.get("grad") else _plain_heads(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind in ("rope", "norm"):
        n, d = case["n"], case["d"]
        elements = n * (case["hq"] + case["hk"]) * d
        size = 4 if case["dtype"] == "f32" else 2
        flops = elements * (3.0 + (math.log2(d) if case["r3"] else 0.0) + (4.0 if kind == "norm" else 0.0) + (8.0 if case.get("grad") else 0.0))
        return {"bytes": float(elements * size * (3 if case.get("grad") else 2) + 8 * n), "flops": flops}
    if kind == "append":
        rows = case["n"] * case["hk"] * 2
        held = case["d"] * 2 if case["bits"] == 16 else case["d"] // 2 + 4
        # rows in, rows held; rows held once more, values out
        return {"bytes": float(rows * (4 * case["d"] + 2 * held) + 16 * case["n"]), "flops": 6.0 * rows * case["d"]}
    b, hk, grp, d = (case[x] for x in ("b", "hk", "group", "d"))
    nodes = _nodes(case)
    length = case["context"] * (0.75 if case["ragged"] else 1.0) + sum(nodes) / b
    positions = b * length
    held = 2 * (d * 2 if case["bits"] == 16 else d // 2 + 4)
    rows = sum(nodes) * hk * grp
    return {"bytes": positions * hk * held + rows * (4.0 * d + 4.0), "flops": 4.0 * d * rows * length}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------------------


def _frequencies64(case):
    s, r = _SCALING[case["scaling"]], case["rot"]
    out = []
    for i in range(r // 2):
        base = s["theta"]
        if case["scaling"] == "ntk" and r > 2:
            base *= math.exp(math.log(s["factor"]) * r / (r - 2.0))
        f = math.exp(-math.log(base) * 2.0 * i / r)
        if case["scaling"] == "linear":
            f /= s["factor"]
        elif case["scaling"] == "bands":
            wave = 2.0 * math.pi / f
            if wave > s["original"] / s["low"]:
                f /= s["factor"]
            elif wave > s["original"] / s["high"]:
                share = (s["original"] / wave - s["low"]) / (s["high"] - s["low"])
                f = (1.0 - share) * f / s["factor"] + share * f
        elif case["scaling"] == "ramp":
            def dim(turns):
                return r * math.log(s["original"] / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))
            lo, hi = max(math.floor(dim(s["high"])), 0), min(math.ceil(dim(s["low"])), r - 1)
            keep = 1.0 - min(max((i - lo) / (hi - lo if hi > lo else 0.001), 0.0), 1.0)
            f = f / s["factor"] * (1.0 - keep) + f * keep
        out.append(f)
    return torch.tensor(out, dtype=torch.float64, device="cuda"), 1.0 + 0.1 * math.log(s["factor"]) if case["scaling"] == "ramp" else 1.0


def _spin64(x, pos, case, way):
    """Pairs as complex numbers, multiplied by amplitude * exp(i way angle)."""
    f, amp = _frequencies64(case)
    z = torch.polar(torch.full((len(pos), len(f)), amp, dtype=torch.float64, device="cuda"), way * pos.double()[:, None] * f)[:, None, :]
    r = case["rot"]
    y = x.clone()
    if case["layout"] == "half":
        w = torch.complex(x[..., : r // 2].contiguous(), x[..., r // 2:r].contiguous()) * z
        y[..., : r // 2], y[..., r // 2:r] = w.real, w.imag
    else:
        w = torch.complex(x[..., 0:r:2].contiguous(), x[..., 1:r:2].contiguous()) * z
        y[..., 0:r:2], y[..., 1:r:2] = w.real, w.imag
    return y


def _butterflies64(x):
    d = x.shape[-1]
    y, h = x, 1
    while h < d:
        v = y.unflatten(-1, (d // (2 * h), 2, h))
        y = torch.stack((v[..., 0, :] + v[..., 1, :], v[..., 0, :] - v[..., 1, :]), dim=-2).flatten(-3)
        h *= 2
    return y / math.sqrt(d)


def _rows64(part, t, d, bits):
    """Values (positions, d) of single rows of one cache plane, from its bytes: numpy on the host would do the same."""
    if bits == 16:
        raw = part.view(torch.int16).to(torch.int32) << 16                                          # planes, t, 64
        raw = raw.view(torch.float32).double()
        place = torch.arange(64, device="cuda")
        place = ((place // 8) ^ (t % 8)[:, None]) * 8 + place % 8
        return torch.cat([raw[i].gather(1, place) for i in range(d // 64)], dim=1)
    word = part.view(torch.int32).long() & 0xFFFFFFFF                                               # t, d / 8
    out = torch.empty(word.shape[0], d, dtype=torch.float64, device="cuda")
    for e in range(8):
        at = (e // 2) if e % 2 == 0 else 4 + e // 2
        out[:, e::8] = ((word >> (4 * at)) & 15).double()
    return out


def _sequence64(cache, table, n, head, case):
    """Keys and values of one sequence's first n positions for one head, 64 bits."""
    p, d, bits = case["page"], case["d"], case["bits"]
    out = []
    pages = table[: -(-n // p)].long()
    blocks = cache[pages, head]
    t = torch.arange(len(pages) * p, device="cuda")
    for i in range(2):
        if bits == 4:
            size = p * d // 2
            codes = _rows64(blocks[:, i * size:(i + 1) * size].reshape(-1, d // 2).contiguous(), t, d, 4)
            rec = blocks[:, 2 * size + i * 4 * p:2 * size + (i + 1) * 4 * p].reshape(-1, 4).contiguous().view(torch.int32).long()[:, 0]
            step = ((rec & 0xFFFF) << 16).to(torch.int32).view(torch.float32).double()
            out.append(((codes - ((rec >> 16) & 0xFFFF).double()[:, None]) * step[:, None])[:n])
        else:
            size = p * d * 2
            part = blocks[:, i * size:(i + 1) * size].reshape(len(pages), d // 64, p, 128).transpose(0, 1).reshape(d // 64, -1, 128)
            out.append(_rows64(part.contiguous(), t, d, 16)[:n])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rope", "norm"):
        dxs, dws = [], []
        for name in ("q", "k"):
            x = s[name].double()
            if kind == "rope":
                if case["inverse"]:
                    x = _spin64(_butterflies64(x) if case["r3"] else x, s["pos"], case, -1.0)
                else:
                    x = _spin64(x, s["pos"], case, 1.0)
                    x = _butterflies64(x) if case["r3"] else x
                dxs.append(x)
                continue
            w = s["w" + name].double()
            size = (x.square().sum(dim=-1, keepdim=True) / case["d"] + s["eps"]).sqrt()
            if not case["grad"]:
                y = _spin64(x / size * w, s["pos"], case, 1.0)
                dxs.append(_butterflies64(y) if case["r3"] else y)
                continue
            g = s["g" + name].double()
            g = _spin64(_butterflies64(g) if case["r3"] else g, s["pos"], case, -1.0)
            dws.append((g * x / size).flatten(0, 1).sum(dim=0))
            g = g * w
            dxs.append(g / size - x * ((g * x).sum(dim=-1, keepdim=True) / case["d"]) / size ** 3)
        return tuple(dxs + dws)
    if kind == "append":
        out = []
        gone = (s["slots"] < 0)[:, None, None]
        for name in ("k", "v"):
            y = s[name].double()
            if case["bits"] == 4:
                c = float(np.float32(case["clip"]))
                top, low = c * y.amax(dim=-1, keepdim=True).clamp(min=0), c * y.amin(dim=-1, keepdim=True).clamp(max=0)
                step = ((top - low) / 15.0).to(torch.float32).to(torch.bfloat16).double()
                step[step < 2.0 ** -100] = 0.0
                zero = torch.round(-low / step)
                y = torch.minimum(torch.maximum(torch.round(y / step), -zero), 15.0 - zero) * step
                y = torch.where(step > 0, y, torch.zeros_like(y))
            out.append(torch.where(gone, torch.zeros_like(y), y))
        return tuple(out)
    hk, grp, d = (case[x] for x in ("hk", "group", "d"))
    starts, context = s["starts"].tolist(), s["contexts"].tolist()
    q = s["q"].double()
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], float("-inf"), dtype=torch.float64, device="cuda")
    for b, (a, e) in enumerate(zip(starts[:-1], starts[1:])):
        n = context[b] + e - a
        seen = torch.ones(e - a, n, dtype=torch.bool, device="cuda")
        for j in range(e - a):
            seen[:, context[b] + j] = (s["mask"][a:e] >> j) & 1 == 1
        for h in range(hk):
            k, v = _sequence64(s["cache"], s["table"][b], n, h, case)
            x = torch.einsum("igd,nd->ign", q[a:e, h * grp:(h + 1) * grp], k) * s["scale"]
            x = x.masked_fill(~seen[:, None, :], float("-inf"))
            lse[a:e, h * grp:(h + 1) * grp] = torch.logsumexp(x, dim=-1)
            o[a:e, h * grp:(h + 1) * grp] = torch.softmax(x, dim=-1) @ v
    return o, lse
