"""Waits of the attention for more than 16 rows a key head that run out: the call ends, tells of it and leaves the process usable."""
import pytest

from tests.test_gpu_kv_cache import Setup, _B, _t

pytestmark = pytest.mark.gpu

STAGE, TILE, PROBABILITIES, SCORES, OUTPUT = 1, 2, 3, 4, 5
TIMEOUT = -8


def _lose(s, ws, out, lse, block, site, index):
    B, torch = _B(), _t()
    d, heads = s.d, s.hk * s.group
    call = B._TREE_CALL.pack(B._TREE_CALL.size, len(s.nodes), s.group, max(s.nodes), d ** -0.5, s.dev["table"].shape[1], s.rows, s.dev["q"].data_ptr(), heads * d, d,
                             out.data_ptr(), heads * d, d, lse.data_ptr(), heads, s.dev["starts"].data_ptr(), s.dev["contexts"].data_ptr(),
                             s.dev["table"].data_ptr(), s.dev["table"].stride(0), s.mask.data_ptr(), ws.data_ptr(), ws.numel())
    return B.load().conqur_debug_tree_attention(s.cache._ref, call, block, site, index, torch.cuda.current_stream().cuda_stream)


def _fresh(s):
    torch = _t()
    return torch.full_like(s.out, 7.0), torch.full_like(s.lse, 7.0)


# Three sequences of 15, 40 and 2 tiles and two key heads: runs of four tiles (three at an end), one item each, so 4 + 4, 10 + 10 and 1 + 1 blocks, the last two
# with a whole item, whose streams have a tile each.
LOST = [(0, TILE, 0), (0, TILE, 1), (0, TILE, 2), (0, TILE, 3), (3, PROBABILITIES, 0), (3, PROBABILITIES, 1), (9, SCORES, 0), (9, SCORES, 1), (0, OUTPUT, 0),
        (0, OUTPUT, 1), (3, OUTPUT, 0), (3, OUTPUT, 1), (28, OUTPUT, 0), (28, OUTPUT, 1), (28, SCORES, 1), (28, PROBABILITIES, 0), (28, TILE, 1)]


def _setup(bits, d):
    s = Setup(91, [900, 2500, 64], [8, 5, 8], 2, 4, d, 32, bits)
    s.run()
    assert _B().conqur_kv_status() == 0
    return s, s.out.clone(), s.lse.clone()


@pytest.mark.parametrize("bits,d", [(4, 128), (16, 128), (4, 64), (16, 64)])
def test_lost_waits_end_the_call_and_are_told_of(bits, d):
    """Whichever warp gives up and whatever is under way then: the kernel ends, the status says so once, and with a zeroed workspace the next call is right."""
    B, torch = _B(), _t()
    s, good, glse = _setup(bits, d)
    ws = B.attention_workspace(s.cache, 4, 8)
    for block, site, index in LOST:
        out, lse = _fresh(s)
        assert _lose(s, ws, out, lse, block, site, index) == 0
        assert B.conqur_kv_status() == TIMEOUT and B.conqur_kv_status() == 0, (block, site, index)
        ws.zero_()
        out, lse = s.run(out=out, lse=lse, workspace=ws)
        assert torch.equal(out, good) and torch.equal(lse, glse) and B.conqur_kv_status() == 0, (block, site, index)
    # barriers that nobody of the run waits for (no stage is used twice; a whole item of two tiles): an ordinary call
    for block, site, index in ((0, STAGE, 1), (28, TILE, 2)):
        out, lse = _fresh(s)
        assert _lose(s, ws, out, lse, block, site, index) == 0 and B.conqur_kv_status() == 0
        assert torch.equal(out, good) and torch.equal(lse, glse)


@pytest.mark.parametrize("bits,d", [(4, 128), (16, 128)])
def test_rows_of_a_lost_wait_are_right_or_left_as_they_were(bits, d):
    """However late the wait runs out, and in one stream only: a row of a head is what an untroubled call gives, or is not touched."""
    B, torch = _B(), _t()
    s, good, glse = _setup(bits, d)
    ws = B.attention_workspace(s.cache, 4, 8)
    for block, site, index in LOST:
        out, lse = _fresh(s)
        ws.zero_()
        assert _lose(s, ws, out, lse, block, site, index) == 0 and B.conqur_kv_status() == TIMEOUT
        right = (out == good).all(dim=-1) & (lse == glse)
        kept = (out == 7.0).all(dim=-1) & (lse == 7.0)
        assert (right | kept)[:21].all(), (block, site, index)
        # the query heads of the item that the block works on, of its sequence's rows, and no others
        rows, heads = slice(0, 8), slice(0, 4)
        if block >= 28:
            rows = slice(13, 21)
        elif block >= 8:
            rows = slice(8, 13)
        want = torch.zeros_like(kept)
        want[rows, heads] = True
        want[21:] = True                                     # (behind the last sequence)
        assert torch.equal(kept, want), (block, site, index)


@pytest.mark.parametrize("bits", [4, 16])
def test_items_before_the_lost_wait_are_written(bits):
    """Runs over several items: those that a block has finished are there, the one it gives up at and its later ones are not."""
    B, torch = _B(), _t()
    n = 200                                                  # 400 items of one tile: runs of four
    s = Setup(92, [40] * n, [9] * n, 2, 2, 128, 16, bits)
    s.run()
    good, glse = s.out.clone(), s.lse.clone()
    ws = B.attention_workspace(s.cache, 2, 9)
    for site, index, items in ((TILE, 0, 4), (TILE, 1, 3), (TILE, 2, 2), (TILE, 3, 1), (OUTPUT, 0, 4), (OUTPUT, 1, 3), (SCORES, 1, 3), (PROBABILITIES, 1, 3)):
        out, lse = _fresh(s)
        ws.zero_()
        assert _lose(s, ws, out, lse, 2, site, index) == 0 and B.conqur_kv_status() == TIMEOUT
        right = (out == good).all(dim=-1) & (lse == glse)
        kept = (out == 7.0).all(dim=-1) & (lse == 7.0)
        lost = kept[: 9 * n].reshape(n, 9, 2, 2)
        assert (right | kept).all() and torch.equal(lost.any(dim=1).any(dim=-1), lost.all(dim=1).all(dim=-1))
        assert int(lost.any(dim=1).any(dim=-1).sum()) == items, (site, index)


@pytest.mark.parametrize("bits", [4, 16])
def test_a_stage_that_is_never_free_ends_the_call(bits):
    """One long item: the warps that bring keys and values give up at the fifth tile."""
    B, torch = _B(), _t()
    s = Setup(93, [64 * 148 * 12], [9], 1, 2, 64, 64, bits)     # a dozen tiles a block
    s.run()
    good, glse = s.out.clone(), s.lse.clone()
    ws = B.attention_workspace(s.cache, 2, 9)
    for index in range(4):
        out, lse = _fresh(s)
        assert _lose(s, ws, out, lse, 100, STAGE, index) == 0 and B.conqur_kv_status() == TIMEOUT
        assert (out == 7.0).all() and (lse == 7.0).all()       # every block has a part of the one item
        ws.zero_()
        out, lse = s.run(out=out, lse=lse, workspace=ws)
        assert torch.equal(out, good) and torch.equal(lse, glse) and B.conqur_kv_status() == 0


def test_two_conditions_are_told_of_one_after_the_other():
    """A time-out and a bad slot, the slot's from another stream and possibly while the status is read: neither is lost."""
    B, torch = _B(), _t()
    s, good, glse = _setup(4, 128)
    ws = B.attention_workspace(s.cache, 4, 8)
    k = torch.randn(1, 2, 128, device="cuda").bfloat16()
    beyond = torch.tensor([10 ** 9], device="cuda")
    side = torch.cuda.Stream()
    for both_first in (True, False, False, False):
        out, lse = _fresh(s)
        ws.zero_()
        assert _lose(s, ws, out, lse, 0, SCORES, 0) == 0
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            B.conqur_kv_append(s.cache, k, k, beyond)
        if both_first:
            side.synchronize()
        assert B.conqur_kv_status() == TIMEOUT
        side.synchronize()
        assert B.conqur_kv_status() == -11 and B.conqur_kv_status() == 0
