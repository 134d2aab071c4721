"""Host logic of the cache and attention calls: sizes and refusals (no device needed; a refused call touches nothing)."""
import ctypes as C

import numpy as np
import pytest

from oracle import kv_oracle as K


@pytest.fixture(scope="module")
def B():
    from paper_2605_10793_b200 import build, binding
    build.build()
    binding.load()
    return binding


P = 1 << 20                                                 # an address that is never dereferenced


def _cache(B, **kw):
    v = dict(page=64, heads=8, d=128, bits=4, clip=1.0, pages=10, ptr=P)
    v.update(kw)
    return B.conqur_kv_cache(v.get("size", C.sizeof(B.conqur_kv_cache)), v["page"], v["heads"], v["d"], v["bits"], v["clip"], v["pages"], v["ptr"])


@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 16])
def test_cache_bytes(B, page, d, bits):
    got = B.load().conqur_kv_cache_bytes(C.byref(_cache(B, page=page, d=d, bits=bits)))
    assert got == 80 * K.block_bytes(page, d, bits)


BAD_CACHES = [dict(size=8), dict(page=0), dict(page=48), dict(page=128), dict(heads=0), dict(heads=65536), dict(d=96), dict(d=256), dict(bits=8),
              dict(clip=-0.5), dict(clip=1.5), dict(clip=float("nan")), dict(pages=0), dict(pages=2 ** 31)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(B, bad):
    lib = B.load()
    c = C.byref(_cache(B, **bad))
    assert lib.conqur_kv_cache_bytes(c) == 0
    assert lib.conqur_kv_append(c, P, 1024, 128, P, 1024, 128, 4, P, None) == -1
    assert lib.conqur_kv_read(c, P, 4, P, P, 1, None) == -1
    assert lib.conqur_tree_attention_workspace_bytes(c, 4, 1) == 0
    assert lib.conqur_tree_attention(c, _tree(B), None) == -1


def test_append_and_read_refusals(B):
    lib = B.load()
    c = C.byref(_cache(B))
    good = [c, P, 1024, 128, P, 1024, 128, 4, P, None]
    for i, bad in ((1, None), (1, P + 1), (4, None), (4, P + 1), (7, -1), (7, 2 ** 29), (8, None), (8, P + 4)):
        args = list(good)
        args[i] = bad
        assert lib.conqur_kv_append(*args) == -1, (i, bad)
    assert lib.conqur_kv_append(C.byref(_cache(B, ptr=None)), *good[1:]) == -1
    assert lib.conqur_kv_append(C.byref(_cache(B, ptr=P + 8)), *good[1:]) == -1
    assert lib.conqur_kv_append(None, *good[1:]) == -1
    assert lib.conqur_kv_append(c, None, 0, 0, None, 0, 0, 0, None, None) == 0                    # no tokens
    good = [c, P, 4, P, P, 1, None]
    for i, bad in ((1, None), (1, P + 4), (2, -1), (3, None), (3, P + 8), (4, P + 2), (5, 2), (5, -1)):
        args = list(good)
        args[i] = bad
        assert lib.conqur_kv_read(*args) == -1, (i, bad)
    assert lib.conqur_kv_read(c, None, 0, None, None, 0, None) == 0


def _tree(B, **kw):
    v = dict(size=B._TREE_CALL.size, batch=2, group=4, nodes=3, scale=0.1, width=5, rows=6, q=P, q_t=4096, q_h=128, o=P, o_t=4096, o_h=128, lse=P, lse_t=32,
             starts=P, contexts=P, table=P, stride=5, mask=P, ws=P, wsb=1 << 30)
    v.update(kw)
    return B._TREE_CALL.pack(*(v[k] for k in ("size", "batch", "group", "nodes", "scale", "width", "rows", "q", "q_t", "q_h", "o", "o_t", "o_h", "lse", "lse_t",
                                              "starts", "contexts", "table", "stride", "mask", "ws", "wsb")))


@pytest.mark.parametrize("bad", [dict(size=8), dict(batch=-1), dict(batch=65536), dict(group=0), dict(group=65), dict(nodes=0), dict(nodes=65),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(width=-1), dict(rows=-1), dict(rows=2 ** 31), dict(q=0),
                                 dict(q=P + 2), dict(q_t=4097), dict(q_h=4), dict(o=0), dict(o=P + 8), dict(o_t=0), dict(o_h=0), dict(o_h=132), dict(lse=P + 2),
                                 dict(starts=0), dict(starts=P + 2), dict(contexts=0), dict(table=0), dict(table=P + 2), dict(stride=-1), dict(mask=P + 4),
                                 dict(ws=0), dict(ws=P + 128)])
def test_attention_refusals(B, bad):
    lib = B.load()
    assert lib.conqur_tree_attention(C.byref(_cache(B)), _tree(B, **bad), None) == -1


def test_attention_sizes(B):
    lib = B.load()
    c = C.byref(_cache(B))
    need = lib.conqur_tree_attention_workspace_bytes(c, 4, 3)
    assert need > 0
    assert lib.conqur_tree_attention(c, _tree(B, wsb=need - 1), None) == -2
    # a workspace for more rows serves fewer
    sizes = [lib.conqur_tree_attention_workspace_bytes(c, g, n) for g, n in ((1, 1), (8, 1), (4, 4), (4, 8), (4, 16), (4, 32), (64, 64))]
    assert sizes == sorted(sizes)
    for g, n in ((0, 1), (65, 1), (1, 0), (1, 65)):
        assert lib.conqur_tree_attention_workspace_bytes(c, g, n) == 0
    assert lib.conqur_tree_attention(c, _tree(B, batch=0), None) == 0 and lib.conqur_tree_attention(c, _tree(B, rows=0), None) == 0
    assert lib.conqur_tree_attention(C.byref(_cache(B, ptr=None)), _tree(B), None) == -1
    assert lib.conqur_tree_attention(c, None, None) == -1
    assert "index" in B.strerror(-11)


def test_oracle_quantiser_is_the_zero_point_quantiser_where_both_signs_occur():
    """Against the fake-quantiser of the calibration oracle (Appendix B): the same codes up to the rounding of the step to bf16."""
    from oracle import conqur_oracle as O
    y = K.bf16(np.random.default_rng(1).standard_normal((200, 128)))
    got = K.values(y, 4)
    ref, _, delta = O.fake_quant_zp(y, 4)
    # a step off by 2^-8 relative moves a value by up to 15 * 2^-8 steps, and one that lies that near a border by one more
    assert np.max(np.abs(got - ref) / delta[:, None]) <= 1 + 16 * 2.0 ** -8
    assert np.mean(np.abs(got - ref) / delta[:, None] > 0.5) < 0.06
    # one-sided and constant rows: 0 is held exactly and the extreme value to half a step
    for row in (np.linspace(1, 3, 128), np.full(128, -2.5), np.zeros(128)):
        row = K.bf16(row)[None]
        c, z, s = K.quantise(row)
        assert (np.abs((c - z) * s - row) <= np.abs(s) / 2 + 15 * 2.0 ** -9 * np.abs(s)).all() and 0 <= z <= 15
