"""CPU checks of rotary positions' C ABI and binding: refusals (no kernel runs) and
frequencies."""
import ctypes
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from paper_2502_21079_amd.positions import _RotaryProblem, _plan

FAKE = ctypes.c_void_p(0x10000)     # aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return ad.load_library()


def _prob(**kw):
    f = kw.pop("freq", (1.0,) * 32)
    p = _RotaryProblem(batch=2, heads=4, kv_heads=2, len=10, head_dim=64, dtype=0, pairs=32, layout=0, axes=1, magnitude=1.0)
    p.axis_pairs[0] = 32
    arr = (ctypes.c_double * max(1, len(f)))(*f)
    p.freq = ctypes.cast(arr, ctypes.POINTER(ctypes.c_double))
    p._arr = arr
    for n, H in (("q", 4), ("k", 2), ("q_out", 4), ("k_out", 2)):
        setattr(p, n + "_stride", (ctypes.c_int64 * 3)(H * 640, 640, 64))
    for k, v in kw.items():
        if k == "axis_pairs":
            v = (ctypes.c_int32 * 4)(*v)
        setattr(p, k, (ctypes.c_int64 * len(v))(*v) if isinstance(v, tuple) else v)
    return p


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), 1), (dict(heads=0), 1), (dict(kv_heads=-1), 1), (dict(len=-1), 1), (dict(dtype=2), 2),
    (dict(head_dim=60), 2), (dict(head_dim=264), 2), (dict(head_dim=0), 2), (dict(pairs=33), 1), (dict(pairs=0), 1),
    (dict(layout=2), 1), (dict(axes=0), 1), (dict(axes=5), 1), (dict(axis_pairs=(31,)), 1),
    (dict(axes=2, axis_pairs=(40, -8)), 1), (dict(magnitude=math.nan), 1), (dict(freq=(1.0,) * 31 + (math.inf,)), 1),
    (dict(heads=65535), 2), (dict(batch=1 << 16, len=1 << 16), 2), (dict(q_stride=(2560, 640, 4)), 1),
    (dict(k_stride=(-8, 640, 64)), 1), (dict(q_out_stride=(0, 640, 64)), 1), (dict(k_out_stride=(1280, 640, 8)), 1),
    (dict(position_stride=(-1, 1)), 1), (dict(axes=2, axis_pairs=(16, 16)), 1),
])
def test_bad_problems_are_refused(lib, kw, status):
    p = _prob(**kw)
    for fn in (lib.adaspa_rotary, lib.adaspa_rotary_bwd):
        assert fn(ctypes.byref(p), FAKE, FAKE, None, 0, None, FAKE, FAKE, None) == status


def test_bad_pointers_are_refused(lib):
    p, off = _prob(), ctypes.c_void_p(0x10008)
    call = lib.adaspa_rotary
    assert call(None, FAKE, FAKE, None, 0, None, FAKE, FAKE, None) == 1
    for bad in (None, off):
        assert call(ctypes.byref(p), bad, FAKE, None, 0, None, FAKE, FAKE, None) == 1
        assert call(ctypes.byref(p), FAKE, bad, None, 0, None, FAKE, FAKE, None) == 1
        assert call(ctypes.byref(p), FAKE, FAKE, None, 0, None, bad, FAKE, None) == 1
        assert call(ctypes.byref(p), FAKE, FAKE, None, 0, None, FAKE, bad, None) == 1
    odd = ctypes.c_void_p(0x10002)
    assert call(ctypes.byref(p), FAKE, FAKE, odd, 0, None, FAKE, FAKE, None) == 1
    assert call(ctypes.byref(p), FAKE, FAKE, None, 0, odd, FAKE, FAKE, None) == 1
    assert call(ctypes.byref(p), FAKE, FAKE, None, 1 << 40, None, FAKE, FAKE, None) == 1
    empty = _prob(len=0)
    assert call(ctypes.byref(empty), None, None, None, 0, None, None, None, None) == 0


def _shape(**kw):
    s = dict(dtype=0, shapes=((2, 4, 10, 64), (2, 2, 10, 64)), strides=((2560, 640, 64, 1), (1280, 640, 64, 1)),
             outs=(None, None), freqs=(1.0,) * 32, layout="half", sections=None, magnitude=1.0, pos_shape=None,
             pos_stride=None)
    s.update(kw)
    return tuple(s.values())


@pytest.mark.parametrize("kw", [
    dict(shapes=((2, 4, 10), (2, 2, 10, 64))), dict(shapes=((2, 4, 10, 64), (2, 2, 11, 64))),
    dict(shapes=((2, 4, 10, 64), (3, 2, 10, 64))), dict(layout="quarter"), dict(freqs=()), dict(freqs=(1.0,) * 33),
    dict(sections=(16, 15)), dict(sections=(8, 8, 8, 4, 4)), dict(sections=(16, 16)),
    dict(strides=((2560, 640, 64, 2), (1280, 640, 64, 1))), dict(strides=((2560, 640, 60, 1), (1280, 640, 64, 1))),
    dict(pos_shape=(9,), pos_stride=(1,)), dict(pos_shape=(3, 10), pos_stride=(10, 1)),
    dict(sections=(16, 16), pos_shape=(2, 10), pos_stride=(10, 1)),
    dict(sections=(16, 16), pos_shape=(2, 10, 2), pos_stride=(20, 1, 10)),
])
def test_bad_arguments_are_refused_by_the_binding(kw):
    _plan(*_shape())
    with pytest.raises(ad.AdaspaError):
        _plan(*_shape(**kw))


def test_tensors_elsewhere_are_refused():
    q = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ad.AdaspaError):
        ad.rotary(q, None, (1.0,))


def test_frequencies():
    f = ad.rotary_frequencies(8, 10000.0)
    assert f == pytest.approx((1.0, 0.1, 0.01, 0.001), rel=1e-15)
    assert ad.rotary_frequencies(8, 10000.0, scaling="linear", factor=4.0) == pytest.approx([x / 4 for x in f], rel=1e-15)
    axes = ad.rotary_frequencies(12, 100.0, sections=(2, 4))
    assert axes == pytest.approx((1.0, 0.1, 1.0, 100 ** -0.25, 100 ** -0.5, 100 ** -0.75), rel=1e-15)
    b = ad.rotary_frequencies(8, 10000.0, scaling="base", factor=8.0)
    assert b[0] == 1.0 and b[-1] == pytest.approx(f[-1] / 8, rel=1e-12)
    # By parts over 4096 positions: 652 turns stay, 0.65 are divided, 65 stay, 6.5 blend.
    p = ad.rotary_frequencies(8, 10000.0, scaling="parts", factor=8.0, context=4096)
    stay = (4096 * 0.01 / (2 * math.pi) - 1) / 31
    assert p == pytest.approx((1.0, 0.1, 0.01 * (stay + (1 - stay) / 8), 0.001 / 8), rel=1e-12)
    assert ad.rotary_magnitude(1.0) == 1.0 and ad.rotary_magnitude(0.5) == 1.0
    assert ad.rotary_magnitude(8.0) == pytest.approx(0.1 * math.log(8.0) + 1)
    for bad in (dict(dims=7), dict(dims=0), dict(dims=8, sections=(1, 2)), dict(dims=8, scaling="more"),
                dict(dims=8, base=0.0), dict(dims=8, factor=-1.0), dict(dims=8, scaling="parts"),
                dict(dims=8, scaling="parts", context=10, low=2.0, high=1.0)):
        with pytest.raises(ad.AdaspaError):
            ad.rotary_frequencies(**bad)
