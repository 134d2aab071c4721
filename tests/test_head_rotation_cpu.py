"""Host logic of the head rotations: frequencies and refusals (no device needed; a refused call touches nothing)."""
import ctypes as C

import numpy as np
import pytest

from oracle import heads_oracle as H


@pytest.fixture(scope="module")
def B():
    from paper_2605_10793_b200 import build, binding
    build.build()
    binding.load()
    return binding


CASES = [dict(), dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=4.0), dict(scaling="ntk", factor=1.0),
         dict(theta=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192),
         dict(theta=10000.0, scaling="ramp", factor=16.0, low=1.0, high=32.0, original=4096),
         dict(theta=10000.0, scaling="ramp", factor=2.0, low=900.0, high=1000.0, original=64)]


@pytest.mark.parametrize("r", [2, 4, 24, 64, 128, 512])
@pytest.mark.parametrize("kw", CASES)
def test_frequencies_follow_the_definition(B, r, kw):
    if r == 2 and kw.get("scaling") == "ntk" and kw["factor"] != 1.0:
        assert B.load().conqur_rope_table_bytes(C.byref(B.rope_config(r, **kw))) == 0
        return
    f, amp = B.conqur_rope_frequencies(B.rope_config(r, **kw))
    want, m = H.frequencies(r, **kw)
    # the oracle's powers and logarithms are good to a few 2^-52 of an exponent of up to 20
    assert np.allclose(f, want, rtol=2.0 ** -46, atol=0) and abs(amp - m) <= 2.0 ** -50
    assert B.load().conqur_rope_table_bytes(C.byref(B.rope_config(r, **kw))) == 8 * (r // 2 + 1)


def test_frequencies_refusals(B):
    lib = B.load()
    good = dict(rotary_dim=64, theta=10000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original=8192)
    assert lib.conqur_rope_table_bytes(C.byref(B.rope_config(**good))) > 0
    nan, inf = float("nan"), float("inf")
    for bad in (dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=514), dict(rotary_dim=-2), dict(theta=1.0), dict(theta=nan), dict(theta=inf),
                dict(factor=0.5), dict(factor=nan), dict(low=0.0), dict(low=4.0), dict(high=nan), dict(high=inf), dict(original=0)):
        cfg = B.rope_config(**{**good, **bad})
        assert lib.conqur_rope_table_bytes(C.byref(cfg)) == 0, bad
        assert lib.conqur_rope_table(C.byref(cfg), 4096, None) == -1, bad
        with pytest.raises(B.ConqurError):
            B.conqur_rope_frequencies(cfg)
    cfg = B.rope_config(**good)
    assert lib.conqur_rope_table(C.byref(cfg), None, None) == -1 and lib.conqur_rope_table(C.byref(cfg), 4100, None) == -1
    cfg.scaling = 5
    assert lib.conqur_rope_table_bytes(C.byref(cfg)) == 0
    cfg = B.rope_config(**good)
    cfg.struct_size = 8
    assert lib.conqur_rope_table_bytes(C.byref(cfg)) == 0 and lib.conqur_rope_table_bytes(None) == 0


def _call(B, **kw):
    p = 1 << 20                                             # never dereferenced: every call below is refused on the host
    v = dict(size=B._HEADS_CALL.size, dtype=1, d=128, rot=128, layout=0, flags=0, wt=1, eps=1e-6, hq=4, hk=2, b=1, t=3, pos=p, pos_b=0, table=p,
             qi=(p, 0, 512, 128), ki=(p, 0, 256, 128), qo=(p, 0, 512, 128), ko=(p, 0, 256, 128), qw=p, kw=p, qg=(p, 0, 512, 128),
             kg=(p, 0, 256, 128), dq=p, dk=p)
    v.update(kw)
    return B._HEADS_CALL.pack(v["size"], v["dtype"], v["d"], v["rot"], v["layout"], v["flags"], v["wt"], v["eps"], v["hq"], v["hk"], v["b"], v["t"],
                              v["pos"], v["pos_b"], v["table"], *v["qi"], *v["ki"], *v["qo"], *v["ko"], v["qw"], v["kw"], *v["qg"], *v["kg"], v["dq"], v["dk"])


REFUSED = [dict(size=100), dict(dtype=2), dict(d=0), dict(d=513), dict(rot=-2), dict(rot=63), dict(rot=130), dict(layout=2), dict(flags=4), dict(hq=0),
           dict(hk=-1), dict(b=-1), dict(t=-1), dict(b=2 ** 20, t=2 ** 20), dict(pos=0), dict(table=0), dict(table=(1 << 20) + 4), dict(d=96, rot=32, flags=1),
           dict(qi=(0, 0, 512, 128)), dict(ko=(0, 0, 256, 128)), dict(qi=((1 << 20) + 1, 0, 512, 128)), dict(qo=(1 << 20, 0, 512, 0)),
           dict(qo=(1 << 20, 0, 0, 128)), dict(b=2, qo=(1 << 20, 0, 512, 128)), dict(pos=(1 << 20) + 4)]


@pytest.mark.parametrize("bad", REFUSED)
def test_head_calls_are_refused(B, bad):
    lib = B.load()
    call = _call(B, **bad)
    assert lib.conqur_rope_heads(call, None) == -1
    assert lib.conqur_norm_rope_heads(call, None) == -1
    assert lib.conqur_norm_rope_heads_backward(call, 1 << 20, 1 << 22, None) == -1


def test_norm_calls_are_refused(B):
    lib = B.load()
    for bad in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(wt=7), dict(flags=2), dict(qw=(1 << 20) + 1)):
        assert lib.conqur_norm_rope_heads(_call(B, **bad), None) == -1, bad
        assert lib.conqur_norm_rope_heads_backward(_call(B, **bad), 1 << 20, 1 << 22, None) == -1, bad
    need = lib.conqur_norm_rope_backward_scratch_bytes(128)
    assert need > 0 and lib.conqur_norm_rope_backward_scratch_bytes(0) == 0 and lib.conqur_norm_rope_backward_scratch_bytes(513) == 0
    assert lib.conqur_norm_rope_heads_backward(_call(B), 1 << 20, need - 1, None) == -2
    assert lib.conqur_norm_rope_heads_backward(_call(B), None, need, None) == -1
    assert lib.conqur_norm_rope_heads_backward(_call(B), (1 << 20) + 8, need, None) == -1
    assert lib.conqur_norm_rope_heads_backward(_call(B, qg=(0, 0, 512, 128)), 1 << 20, need, None) == -1
    assert lib.conqur_rope_heads(None, None) == -1
    assert lib.conqur_rope_heads(_call(B, t=0), None) == 0 and lib.conqur_norm_rope_heads(_call(B, b=0), None) == 0       # no tokens: nothing to do
