"""Host-only checks of the norm + rotation entry points: refusals before any launch, legal no-ops, the axis helper."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_14498_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2608_14498_b200 import build

    build.build()
    return B.load_library()


def desc(hq=4, hkv=2, d=128, rot=128, axes=1, pair_axis=None, eps=1e-6, dtype=B.RPX_BF16):
    return B.RopeDesc(hq, hkv, d, rot, axes, pair_axis, eps, dtype)


def forward(lib, dsc, q=0x1000, k=0x1000, qs=512, ks=256, wq=0x1000, wk=0x1000, pos=0x1000, pstride=16, inv=0x1000, n=16,
            qo=0x1000, ko=0x1000, qos=512, kos=256):
    return lib.rpx_qk_norm_rope(ctypes.byref(dsc) if dsc is not None else None, q, k, qs, ks, wq, wk, pos, pstride, inv, n, qo,
                                ko, qos, kos, None)


def backward(lib, dsc, dq=0x1000, dk=0x1000, n=16, wq=0x1000, wk=0x1000, dwq=0x1000, dwk=0x1000, ws=0x1000, ws_bytes=1 << 24):
    return lib.rpx_qk_norm_rope_backward(ctypes.byref(dsc), 0x1000, 0x1000, 512, 256, wq, wk, 0x1000, 16, 0x1000, dq, dk, n,
                                         0x1000, 0x1000, 512, 256, dwq, dwk, 0, ws, ws_bytes, None)


def test_forward_refusals(lib):
    assert forward(lib, None) == -1
    for bad in (dict(hq=0), dict(hkv=-1), dict(d=96), dict(rot=8), dict(rot=120), dict(rot=144), dict(axes=0), dict(axes=9),
                dict(eps=-1.0), dict(eps=float("nan")), dict(pair_axis=b"\0" * 63 + b"\1")):
        assert forward(lib, desc(**bad)) == -2, bad
    assert forward(lib, desc(dtype=5)) == -3
    for bad in (dict(q=None), dict(k=None), dict(pos=None), dict(inv=None), dict(qo=None), dict(ko=None), dict(wq=None),
                dict(wk=None)):
        assert forward(lib, desc(), **bad) == -1, bad
    for bad in (dict(qs=504), dict(ks=128), dict(qos=504), dict(kos=248), dict(pstride=15), dict(n=-1)):
        assert forward(lib, desc(), **bad) == -2, bad
    for bad in (dict(qs=516), dict(kos=260), dict(q=0x1008), dict(wk=0x1004), dict(ko=0x1002)):
        assert forward(lib, desc(), **bad) == -4, bad
    assert forward(lib, desc(), q=None, k=None, pos=None, n=0) == 0  # nothing to do


def test_backward_refusals(lib):
    assert backward(lib, desc(), dq=None) == -1
    assert backward(lib, desc(), dk=0x1008) == -4
    assert backward(lib, desc(), dwq=None) == -1                      # one weight gradient without the other
    assert backward(lib, desc(), wq=None, wk=None) == -1              # a weight gradient without weights
    assert backward(lib, desc(), ws=None) == -5
    assert backward(lib, desc(), ws_bytes=256) == -5
    assert backward(lib, desc(), ws=0x1010) == -4
    assert backward(lib, desc(), wq=None, wk=None, dwq=None, dwk=None, ws=None, ws_bytes=0, n=0) == 0


def test_pair_axis_helper():
    assert B.mrope_pair_axis([2, 3, 3]) == [0, 0, 1, 1, 1, 2, 2, 2]
    assert B.mrope_pair_axis([4, 2, 2], interleaved=True) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert B.mrope_pair_axis([5]) == [0] * 5
    with pytest.raises(ValueError):
        B.mrope_pair_axis([1, 3], interleaved=True)
    with pytest.raises(ValueError):
        B.mrope_pair_axis([])


def test_wrapper_checks():
    q, k = torch.zeros(3, 4, 64).bfloat16(), torch.zeros(3, 2, 64).bfloat16()
    pos, inv = torch.zeros(3, dtype=torch.int32), torch.ones(32)

    def make(**kw):
        a = dict(q=q, k=k, positions=pos, inv_freq=inv, q_weight=None, k_weight=None, pair_axis=None, eps=1e-6)
        a.update(kw)
        return B._rope_desc(**a)

    assert make().rot_dim == 64
    for bad in (dict(k=k.float()), dict(positions=pos.long()), dict(inv_freq=inv.double()), dict(q_weight=torch.ones(64))):
        with pytest.raises(TypeError):
            make(**bad)
    for bad in (dict(k=torch.zeros(4, 2, 64).bfloat16()), dict(positions=pos[:2]), dict(pair_axis=[0] * 31),
                dict(q_weight=torch.ones(32).bfloat16()), dict(positions=torch.zeros(3, 2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            make(**bad)


@pytest.mark.parametrize("make", [list, tuple, bytes, bytearray, iter, np.array, lambda a: np.array(a, dtype=np.int32),
                                  lambda a: np.array(a, dtype=np.uint8), lambda a: np.array(sum(([x, 9] for x in a), []))[::2],
                                  torch.tensor, lambda a: torch.tensor(a, dtype=torch.uint8),
                                  lambda a: [np.int64(x) for x in a]])
def test_pair_axis_means_its_numbers(make):
    """Every kind of sequence gives the kernel the same axis per pair (an array's memory holds more bytes than numbers)."""
    q, k = torch.zeros(3, 4, 64).bfloat16(), torch.zeros(3, 2, 64).bfloat16()
    want = B.mrope_pair_axis([8, 12, 12])
    desc = B._rope_desc(q, k, torch.zeros(3, 3, dtype=torch.int32), torch.ones(32), None, None, make(want), 1e-6)
    at = ctypes.c_void_p.from_buffer(desc, B.RopeDesc.pair_axis.offset).value
    assert list(ctypes.string_at(at, 32)) == want


def test_pair_axis_refusals():
    q, k = torch.zeros(3, 4, 64).bfloat16(), torch.zeros(3, 2, 64).bfloat16()

    def make(axes):
        return B._rope_desc(q, k, torch.zeros(3, 3, dtype=torch.int32), torch.ones(32), None, None, axes, 1e-6)

    for bad in ([-1] + [0] * 31, np.full(32, -1), np.full(32, 256), np.zeros(31, np.int64), torch.zeros(64, dtype=torch.int32)):
        with pytest.raises(ValueError):
            make(bad)
    for bad in ([0.5] * 32, np.zeros(32), np.zeros((32, 2), np.int64), "a" * 32):
        with pytest.raises(TypeError):
            make(bad)
