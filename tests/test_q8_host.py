"""The 8-bit cache's argument checks (no GPU), and pins of its 64-bit statement in oracle/q8.py."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import q8
from paper_2505_00570_b200 import binding as fk

K, V, KS, VS = 0x10000000, 0x20000000, 0x30000000, 0x34000000   # never dereferenced by the checks
NK, NV = 0x40000000, 0x50000000


def lay(kind=fk.Q8_E4M3, B=1, L=2, H=2, cap=256, hd=128, block=64):
    return fk.Q8Layout(kind, B, L, H, cap, hd, block, L * H * cap * hd, H * cap * hd, cap * hd, hd)


def check(layout, lens, k=K, v=V, ks=KS, vs=VS, nk=NK, nv=NV, dtype=fk.BF16, n=1):
    return fk.lib().freqkv_check_append_q8(ctypes.byref(layout), k, v, ks, vs, nk, nv, dtype, n, (ctypes.c_int32 * len(lens))(*lens))


def test_check_append_q8():
    assert check(lay(), [0]) == fk.OK
    assert check(lay(), [255]) == fk.OK
    assert check(lay(), [256]) == fk.ERR_CAPACITY
    assert check(lay(), [200], n=57) == fk.ERR_CAPACITY
    assert check(lay(), [257]) == fk.ERR_INVALID_ARG
    assert check(lay(), [-1]) == fk.ERR_INVALID_ARG
    assert check(lay(), [0], n=-1) == fk.ERR_INVALID_ARG
    assert check(lay(), [0], n=0, nk=0, nv=0) == fk.OK
    assert check(lay(), [0], nk=0) == fk.ERR_INVALID_ARG
    assert check(lay(), [0], nk=NK + 8) == fk.ERR_UNSUPPORTED
    assert check(lay(), [0], dtype=7) == fk.ERR_UNSUPPORTED
    assert check(lay(B=2), [3, 4], dtype=fk.F32) == fk.OK


def test_check_q8_layout():
    for block in (16, 32, 64, 128):
        assert check(lay(block=block), [0]) == fk.OK
    for block in (0, 8, 24, 48, 256, -64):
        assert check(lay(block=block), [0]) == fk.ERR_UNSUPPORTED
    assert check(lay(kind=2), [0]) == fk.ERR_UNSUPPORTED
    assert check(lay(hd=120), [0]) == fk.ERR_UNSUPPORTED          # rows would not stay 16-byte aligned
    assert check(lay(hd=272), [0]) == fk.ERR_UNSUPPORTED
    assert check(lay(hd=16), [0]) == fk.OK
    assert check(lay(cap=0), [0]) == fk.ERR_INVALID_ARG
    bad = lay()
    bad.stride_token = 136                                         # a multiple of 8 only
    assert check(bad, [0]) == fk.ERR_UNSUPPORTED
    bad = lay()
    bad.stride_head = 128 * 100                                    # heads overlap
    assert check(bad, [0]) == fk.ERR_UNSUPPORTED
    assert fk.lib().freqkv_check_append_q8(None, K, V, KS, VS, NK, NV, fk.BF16, 1, (ctypes.c_int32 * 1)(0)) == fk.ERR_INVALID_ARG
    assert fk.lib().freqkv_check_append_q8(ctypes.byref(lay()), K, V, KS, VS, NK, NV, fk.BF16, 1, None) == fk.ERR_INVALID_ARG


def test_check_q8_pointers():
    for name in ("k", "v", "ks", "vs"):
        assert check(lay(), [0], **{name: 0}) == fk.ERR_INVALID_ARG
    assert check(lay(), [0], k=K + 8) == fk.ERR_UNSUPPORTED
    assert check(lay(), [0], ks=KS + 2) == fk.ERR_UNSUPPORTED
    assert check(lay(), [0], ks=KS + 4) == fk.OK
    assert check(lay(), [0], v=K) == fk.ERR_INVALID_ARG
    assert check(lay(), [0], v=K + 4096) == fk.ERR_INVALID_ARG     # overlap
    assert check(lay(), [0], ks=K + 128) == fk.ERR_INVALID_ARG     # scales inside the codes
    assert check(lay(), [0], vs=KS + 16) == fk.ERR_INVALID_ARG


def test_check_quantize():
    def quantize(src, layout, lens, ks=K, vs=V):
        return fk.lib().freqkv_check_quantize(ctypes.byref(src), NK, NV, (ctypes.c_int32 * len(lens))(*lens), ctypes.byref(layout), ks, vs, KS, VS)

    def src(dtype=fk.BF16, B=1, L=2, H=2, cap=200, hd=128):
        st, out = fk.layout_contiguous(dtype, B, L, H, cap, hd)
        assert st == fk.OK
        return out

    assert quantize(src(), lay(), [200]) == fk.OK
    assert quantize(src(dtype=fk.F32), lay(), [0]) == fk.OK
    assert quantize(src(), lay(), [201]) == fk.ERR_INVALID_ARG            # more rows than the source has
    assert quantize(src(cap=300), lay(), [257]) == fk.ERR_INVALID_ARG     # more than the cache holds
    assert quantize(src(), lay(), [-1]) == fk.ERR_INVALID_ARG
    assert quantize(src(L=3), lay(), [10]) == fk.ERR_INVALID_ARG
    assert quantize(src(hd=64), lay(), [10]) == fk.ERR_INVALID_ARG
    assert quantize(src(), lay(), [10], ks=NK) == fk.ERR_INVALID_ARG      # codes over the source


def test_check_attend_q8():
    Q, O = NK, NV

    def check_attend(layout, lens, layer=0, q=Q, out=O, G=1, n_new=1):
        return fk.lib().freqkv_check_attend_q8(ctypes.byref(layout), K, V, KS, VS, layer, q, out, G, n_new, (ctypes.c_int32 * len(lens))(*lens))

    assert check_attend(lay(B=2), [1, 256]) == fk.OK
    for G in (1, 3, 8, 9, 64):
        assert check_attend(lay(), [10], G=G) == fk.OK
    assert check_attend(lay(), [10], G=65) == fk.ERR_UNSUPPORTED
    assert check_attend(lay(), [10], G=0) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [0]) == fk.ERR_INVALID_ARG            # an empty cache has nothing to attend to
    assert check_attend(lay(), [257]) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], layer=2) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], layer=-1) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], q=0) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], out=Q) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], q=Q + 2) == fk.ERR_UNSUPPORTED
    assert check_attend(lay(hd=64), [10]) == fk.ERR_UNSUPPORTED
    assert check_attend(lay(), [10], n_new=0) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], n_new=11) == fk.ERR_INVALID_ARG
    assert check_attend(lay(), [10], n_new=10) == fk.OK


def test_null_context_and_binding_checks():
    one = (ctypes.c_int32 * 1)(0)
    lib, layout = fk.lib(), lay()
    assert lib.freqkv_append_q8(None, ctypes.byref(layout), K, V, KS, VS, NK, NV, fk.BF16, 1, one, None) == fk.ERR_INVALID_ARG
    st, src = fk.layout_contiguous(fk.BF16, 1, 2, 2, 256, 128)
    assert lib.freqkv_quantize(None, ctypes.byref(src), NK, NV, one, ctypes.byref(layout), K, V, KS, VS, None) == fk.ERR_INVALID_ARG
    assert lib.freqkv_dequantize(None, ctypes.byref(layout), K, V, KS, VS, one, ctypes.byref(src), NK, NV, None) == fk.ERR_INVALID_ARG
    c = fk.Q8Cache.empty(1, 2, 2, 100, kind=fk.Q8_INT8, block_tokens=32, device="cpu")
    assert tuple(c.k_scale.shape) == (1, 2, 2, 4) and c.layout.kind == fk.Q8_INT8
    with pytest.raises(fk.FreqKVError):
        fk.Q8Cache(c.k, c.v, c.k_scale, c.v_scale, 64)             # scales of another block size
    with pytest.raises(fk.FreqKVError):
        fk.Q8Cache(c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale, 32)
    with pytest.raises(fk.FreqKVError):
        fk.Q8Cache(c.k, c.v[..., :64], c.k_scale, c.v_scale, 32)


def test_oracle_codes_against_torch_and_closed_forms():
    rng = np.random.default_rng(4)
    x = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.integers(-4, 3, 4000), np.arange(-1000, 1000) / 512.0, [0.0, 448.0, -448.0, 464.0]])
    x = np.clip(x, -448, 448)
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(q8.codes(x.astype(np.float32), 1.0, q8.E4M3), want)
    assert q8.scale(448.0, q8.E4M3) == 1.0 and q8.scale(449.0, q8.E4M3) == 2.0 and q8.scale(224.0, q8.E4M3) == 0.5
    assert q8.scale(127.0, q8.INT8) == 1.0 and q8.scale(0.0, q8.INT8) == 0.0 and q8.scale(1e-44, q8.INT8) == 2.0 ** -126
    assert list(q8.codes([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 300.0, np.inf, -np.inf, np.nan], 1.0, q8.INT8)) == [0, 2, 2, 0, -2, 126, 127, 127, -127, 0]
    # a block that grows: one row of ones, then a row of twos
    c, s = q8.append(np.zeros((16, 2)), np.zeros(1), [[1.0, -1.0]], 0, q8.INT8, 16)
    c, s = q8.append(c, s, [[2.0, 0.0]], 1, q8.INT8, 16)
    assert list(c[0]) == [64, -64] and list(c[1]) == [127, 0]      # 127 / 2 = 63.5, to even
