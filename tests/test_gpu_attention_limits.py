"""Attention over the cache at the limits of its arguments."""
import time

import numpy as np
import pytest

from oracle import kv_oracle as K
from tests.test_gpu_kv_cache import Setup, _B, _codes_bound, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hk,group", [(2, 2), (1, 4), (2, 16)])
def test_a_context_beyond_its_table_sees_the_table_and_costs_no_more(hk, group, bits):
    """Positions without a place in the table are not seen, however many the context claims: the work is that of the table, not of 2^24 tiles."""
    B, torch = _B(), _t()
    s = Setup(101, [204, 205, 12], [4, 3, 2], hk, group, 128, 16, bits)       # the first two fill their 13 pages, and so the table
    good, glse = (x.clone() for x in s.run())
    s.check(good, glse)
    ws = B.attention_workspace(s.cache, group, 4)
    for claim in (205, 300, 2 ** 30, 2 ** 31 - 1):
        s.dev["contexts"][0] = claim
        times = []
        for _ in range(3):                                   # (the best of three: the host may be busy)
            torch.cuda.synchronize()
            begin = time.perf_counter()
            out, lse = s.run(out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0), workspace=ws)
            assert B.conqur_kv_status() == -11
            times.append(time.perf_counter() - begin)
        assert min(times) < 0.1
        assert torch.equal(out[4:], good[4:]) and torch.equal(lse[4:], glse[4:])
        # its drafted tokens lie at `claim` and behind: those past position 207 have no place; the others see by their masks
        seen = np.zeros((4, 208), bool)
        seen[:, :claim] = True
        for i in range(4):
            for j in range(4):
                if claim + j < 208:
                    seen[i, claim + j] = (s.masks[0][i] >> j) & 1
        for h in range(hk * group):
            kh = h // group
            want, wl, mass, size = K.attend(s.q[:4, h], s.k[0][:, kh], s.v[0][:, kh], seen, 128 ** -0.5)
            delta = 2.0 ** -18 * size
            bound = (2.0 ** -8 + 2 * delta[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want) + 1e-30
            bound += _codes_bound(s.step[0][:, kh], s.k[0][:, kh], s.q[:4, h], seen, 128 ** -0.5)
            assert (np.abs(out[:4, h].float().cpu().numpy() - want) <= bound).all(), (claim, h)
            assert (np.abs(lse[:4, h].cpu().numpy() - wl) <= delta + 2.0 ** -20 * np.abs(wl) + 2.0 ** -13).all()
    # no table at all: nothing is seen
    s.dev["table"] = s.dev["table"][:, :0]
    out, lse = s.run(out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0), workspace=ws)
    assert B.conqur_kv_status() == -11 and not out[:9].any() and torch.isneginf(lse[:9]).all() and (out[9:] == 7.0).all()


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hk,group,d", [(2, 2, 64), (1, 4, 128), (2, 10, 128), (1, 20, 64)])
def test_tokens_behind_max_nodes_are_nan_and_told_of(hk, group, d, bits):
    """A call whose max_nodes (1 unless given) is too small: no row of a sequence is left unwritten, and the rows that are computed are right."""
    B, torch = _B(), _t()
    s = Setup(102, [70] * 40 + [5], [1] * 39 + [5, 1], hk, group, d, 16, bits, kind="chain")
    s.masks[39] = [1] * 5
    s.mask[39:44] = 1
    good, glse = (x.clone() for x in s.run(max_nodes=5))
    for args in (dict(out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0)), dict(out=None, lse=None)):
        out, lse = s.run(max_nodes=1, **args)
        assert B.conqur_kv_status() == -11
        assert torch.isnan(out[40:44]).all() and torch.isnan(lse[40:44]).all()
        if args["out"] is not None:
            out[40:44], lse[40:44] = good[40:44], glse[40:44]
            s.check(out, lse)
    # two at the most: the second of the long one is there, too
    out, lse = s.run(max_nodes=2, out=torch.full_like(good, 7.0), lse=torch.full_like(glse, 7.0))
    assert B.conqur_kv_status() == -11 and torch.isnan(out[41:44]).all() and torch.isnan(lse[41:44]).all()
    out[41:44], lse[41:44] = good[41:44], glse[41:44]
    s.check(out, lse)
    # without lse, into strided rows: nothing beside them is touched
    wide = torch.full((s.rows, hk * group + 1, d + 8), 7.0, device="cuda").bfloat16()
    s.run(max_nodes=1, out=wide[:, 1:, :d])
    assert B.conqur_kv_status() == -11 and torch.isnan(wide[40:44, 1:, :d]).all()
    assert (wide[..., d:] == 7.0).all() and (wide[:, 0] == 7.0).all() and (wide[45:] == 7.0).all()
    # thousands of tokens where one was meant, and spans that leave q: those sequences are left out
    n = 3000
    q = torch.randn(n, hk * group, d, device="cuda").bfloat16()
    one = dict(contexts=s.dev["contexts"][:1], table=s.dev["table"][:1])
    ws = B.attention_workspace(s.cache, group, 1)
    out, lse = B.conqur_tree_attention(q, s.cache, torch.tensor([0, n], dtype=torch.int32, device="cuda"), workspace=ws, **one)
    assert B.conqur_kv_status() == -11 and torch.isfinite(out[0]).all() and torch.isnan(out[1:]).all() and torch.isnan(lse[1:]).all()
    for span in ([0, n + 1], [-1, n], [5, 3]):
        o, l = torch.full_like(q, 7.0), torch.full_like(lse, 7.0)
        B.conqur_tree_attention(q, s.cache, torch.tensor(span, dtype=torch.int32, device="cuda"), workspace=ws, out=o, lse=l, **one)
        assert B.conqur_kv_status() == -11 and (o == 7.0).all() and (l == 7.0).all()


@pytest.mark.parametrize("hk,group,nodes", [(2, 1, 1), (2, 4, 1), (1, 4, 3), (2, 8, 2), (2, 8, 4), (1, 16, 20)])
@pytest.mark.parametrize("context,low", [(0, (0, 1)), (90, (0, 64)), (300, (0, 300)), (300, (32, 64)), (9000, (0, 8990)), (9000, (100, 9000))])
def test_scores_of_minus_infinity_weigh_nothing(context, low, hk, group, nodes):
    """Keys with an element of -inf that every query meets with a positive one: weight 0, also where a warp, a stream or a part of an item has met no other."""
    B, torch = _B(), _t()
    d, page = 128, 32
    s = Setup(103, [context, 33], [nodes, 1], hk, group, d, page, 16, kind="chain")
    s.q[..., 5] = np.abs(s.q[..., 5]) + 0.5
    s.q = K.bf16(s.q)
    s.dev["q"] = torch.from_numpy(s.q.astype(np.float32)).cuda().bfloat16()
    at = torch.arange(*low, device="cuda")
    k, v = (torch.from_numpy(x[0][low[0]:low[1]].astype(np.float32)).cuda().bfloat16() for x in (s.k, s.v))
    k[..., 5] = float("-inf")
    B.conqur_kv_append(s.cache, k, v, s.dev["table"][0].long()[at // page] * page + at % page)
    out, lse = s.run()
    assert B.conqur_kv_status() == 0
    seen = np.ones((nodes, context + nodes), bool)
    for i in range(nodes):
        seen[i, context + i + 1:] = False
    seen[:, low[0]:low[1]] = False                           # what weighs nothing might as well not be seen
    for h in range(hk * group):
        want, wl, mass, size = K.attend(s.q[:nodes, h], s.k[0][:, h // group], s.v[0][:, h // group], seen, d ** -0.5)
        delta = 2.0 ** -18 * size
        bound = (2.0 ** -8 + 2 * delta[:, None] + 2.0 ** -19) * mass + 2.0 ** -8 * np.abs(want) + 1e-30
        assert (np.abs(out[:nodes, h].float().cpu().numpy() - want) <= bound).all(), h
        got, none = lse[:nodes, h].cpu().numpy().astype(np.float64), np.isneginf(wl)
        assert np.array_equal(np.isneginf(got), none)
        assert (np.abs(got[~none] - wl[~none]) <= (delta + 2.0 ** -20 * np.abs(wl) + 2.0 ** -13)[~none]).all()
