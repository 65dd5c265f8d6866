"""Argument checks of eviction by attention weight (no GPU), and pins of its 64-bit statement."""
import ctypes

import numpy as np

from oracle import evict as oe
from oracle import attention as oa
from paper_2505_00570_b200 import binding as fk

K, V, M, MO, R = 0x10000000, 0x20000000, 0x30000000, 0x31000000, 0x32000000   # never dereferenced


def lay(dtype=fk.BF16, B=2, L=2, H=2, cap=256, hd=128):
    st, out = fk.layout_contiguous(dtype, B, L, H, cap, hd)
    assert st == fk.OK
    return out


def check(lens, kept, sink=4, recent=8, k=K, v=V, m=M, mo=MO, r=R, layout=None):
    layout = layout or lay()
    c = (ctypes.c_int32 * len(lens))(*lens) if lens else None
    return fk.lib().freqkv_check_evict(ctypes.byref(layout), k, v, m, mo, r, c, (ctypes.c_int32 * len(kept))(*kept) if kept else None, sink, recent)


def test_check_evict():
    assert check([256, 100], [126, 50]) == fk.OK
    assert check([256, 100], [252, 96]) == fk.OK                  # everything stays
    assert check([256, 12], [8, 8]) == fk.OK                      # sinks and recent rows only
    assert check([256, 4], [0, 0], recent=0) == fk.OK             # sinks only
    assert check([0, 0], [0, 0], sink=0, recent=0) == fk.OK       # nothing there
    assert check([257, 100], [126, 50]) == fk.ERR_INVALID_ARG
    assert check([256, 3], [126, 0], recent=0) == fk.ERR_INVALID_ARG    # fewer rows than sinks
    assert check([256, 100], [7, 50]) == fk.ERR_INVALID_ARG       # fewer than the recent rows
    assert check([256, 100], [253, 50]) == fk.ERR_INVALID_ARG     # more than there are
    assert check([256, 100], [126, 50], sink=-1) == fk.ERR_INVALID_ARG
    assert check([256, 100], [126, 50], recent=-1) == fk.ERR_INVALID_ARG
    assert check(None, [1, 1]) == fk.ERR_INVALID_ARG and check([9, 9], None) == fk.ERR_INVALID_ARG


def test_check_evict_pointers():
    ok = ([256, 100], [126, 50])
    for name in ("k", "v", "m", "mo"):
        assert check(*ok, **{name: 0}) == fk.ERR_INVALID_ARG
    assert check(*ok, r=0) == fk.OK
    assert check(*ok, mo=M) == fk.OK                              # in place
    assert check(*ok, mo=M + 4) == fk.ERR_INVALID_ARG             # half over itself
    assert check(*ok, m=K + 64) == fk.ERR_INVALID_ARG
    assert check(*ok, r=M) == fk.ERR_INVALID_ARG
    assert check(*ok, r=V + 4096) == fk.ERR_INVALID_ARG
    assert check(*ok, m=M + 2) == fk.ERR_UNSUPPORTED
    assert check(*ok, r=R + 1) == fk.ERR_UNSUPPORTED
    assert check(*ok, k=K + 8) == fk.ERR_UNSUPPORTED
    for hd in (8, 80, 256):
        assert check(*ok, layout=lay(hd=hd, dtype=fk.F32)) == fk.OK


def test_check_attend_mass():
    def mass(lens=(10, 64), layer=0, k=K, q=V, m=M, G=2, n=5, layout=None):
        return fk.lib().freqkv_check_attend_mass(ctypes.byref(layout or lay()), k, layer, q, m, G, n, (ctypes.c_int32 * 2)(*lens))

    assert mass() == fk.OK
    assert mass(G=64) == fk.OK and mass(G=65) == fk.ERR_UNSUPPORTED and mass(G=0) == fk.ERR_INVALID_ARG
    assert mass(n=0) == fk.ERR_INVALID_ARG and mass(n=11) == fk.ERR_INVALID_ARG and mass(n=10) == fk.OK
    assert mass(lens=(10, 257)) == fk.ERR_INVALID_ARG
    assert mass(layer=2) == fk.ERR_INVALID_ARG and mass(layer=-1) == fk.ERR_INVALID_ARG
    for name in ("k", "q", "m"):
        assert mass(**{name: 0}) == fk.ERR_INVALID_ARG
    assert mass(k=K + 8) == fk.ERR_UNSUPPORTED and mass(m=M + 2) == fk.ERR_UNSUPPORTED
    assert mass(layout=lay(dtype=fk.F32)) == fk.ERR_UNSUPPORTED and mass(layout=lay(hd=64)) == fk.ERR_UNSUPPORTED


def test_null_context():
    lib, layout, one = fk.lib(), lay(B=1), (ctypes.c_int32 * 1)(100)
    assert lib.freqkv_evict(None, ctypes.byref(layout), K, V, M, M, None, one, one, 4, 8, None) == fk.ERR_INVALID_ARG
    assert lib.freqkv_attend_decode_mass(None, ctypes.byref(layout), K, V, 0, M, MO, R, 1, one, 0.0, 0.0, None) == fk.ERR_INVALID_ARG


def test_oracle_weights_and_keep():
    rng = np.random.default_rng(3)
    k, q = rng.normal(size=(40, 16)), rng.normal(size=(2, 5, 16))
    w = oe.weights(q, k, 40, 100.0)
    assert np.isclose(w.sum(), 10)                                # every token of every head gives away one
    one = oe.weights(q[:, 4:], k, 40, 100.0)
    v = np.eye(40, 16)                                            # values that read the first 16 weights off
    assert np.allclose(oa.attend_decode(q[:, 4], k, v, 40, 100.0).sum(0), one[:16])
    assert np.allclose(oe.weights(np.zeros((1, 3, 16)), k, 4, 0.0), [1 / 2 + 1 / 3 + 1 / 4, 1 / 2 + 1 / 3 + 1 / 4, 1 / 3 + 1 / 4, 1 / 4])
    m = np.array([9.0, 1.0, 5.0, 5.0, -0.0, 0.0, np.nan, 7.0, 5.0, -np.inf])
    assert oe.keep(m, 10, 4, 1, 1) == [0, 2, 6, 7, 9]             # NaN, 7, then the first of three fives
    assert oe.keep(m, 9, 6, 0, 0) == [0, 2, 3, 6, 7, 8]
    assert oe.keep(m, 6, 5, 0, 0) == [0, 1, 2, 3, 4]              # the zeros are equal
