"""CPU checks of the 8-bit cache's C ABI and binding: refusals (no kernel runs), and
the 64-bit definitions against torch's own conversion."""
import ctypes
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from paper_2502_21079_amd.cache import _Cache, _CacheProblem, _plan, _pool
from _cache_ref import E4M3, Sequences, least_scale, nearest, value_of_code

FAKE = ctypes.c_void_p(0x10000)     # aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return ad.load_library()


def _prob(**kw):
    p = _CacheProblem(batch=2, heads=2, kv_heads=2, len=10, head_dim=64, dtype=0, pages=8, page=16, max_pages=4, causal=1,
                      softmax_scale=0.0, table_stride=4)
    for n in ("q", "out", "k", "v"):
        setattr(p, n + "_stride", (ctypes.c_int64 * 3)(1280, 640, 64))
    for k, v in kw.items():
        setattr(p, k, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return p


def _cache(**kw):
    c = _Cache(*[FAKE.value] * 5)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _calls(lib, p, c):
    p, c = p and ctypes.byref(p), c and ctypes.byref(c)
    return (lib.adaspa_cache_write(p, c, FAKE, FAKE, FAKE, None, None),
            lib.adaspa_cache_read(p, c, FAKE, None, FAKE, FAKE, None),
            lib.adaspa_cache_attn(p, c, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1 << 40, None))


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), 1), (dict(heads=0, kv_heads=0), 1), (dict(kv_heads=0), 1), (dict(len=-1), 1), (dict(pages=-1), 1),
    (dict(max_pages=-1), 1), (dict(table_stride=-1), 1), (dict(softmax_scale=math.inf), 1), (dict(dtype=2), 2),
    (dict(head_dim=96), 2), (dict(head_dim=256), 2), (dict(page=8), 2), (dict(page=48), 2), (dict(page=256), 2),
    (dict(batch=40000), 2), (dict(heads=40000, kv_heads=40000, batch=1), 2), (dict(len=1 << 28), 2),
    (dict(max_pages=1 << 24), 2),
])
def test_bad_problems_are_refused(lib, kw, status):
    p = _prob(**kw)
    assert _calls(lib, p, _cache()) == (status,) * 3
    assert lib.adaspa_cache_attn_workspace(ctypes.byref(p)) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q_stride=(1280, 640, 4)), (0, 0, 1)), (dict(q_stride=(-8, 640, 64)), (0, 0, 1)),
    (dict(out_stride=(0, 640, 64)), (0, 0, 1)), (dict(out_stride=(1280, 640, 32)), (0, 0, 1)),
    (dict(k_stride=(1280, 4, 64)), (1, 1, 0)), (dict(v_stride=(1280, 640, -64)), (1, 1, 0)),
    (dict(k_stride=(0, 640, 64)), (0, 1, 0)), (dict(v_stride=(1280, 640, 8)), (0, 1, 0)),
])
def test_bad_strides_are_refused(lib, kw, status):
    p, c = _prob(**kw), _cache()
    for fn, st in zip(("write", "read", "attn"), status):
        if st:
            got = dict(zip(("write", "read", "attn"), _calls_of(lib, p, c, fn)))
            assert got[fn] == st


def _calls_of(lib, p, c, which):
    """Only the call that is expected to be refused (the others would be launched)."""
    p, c = ctypes.byref(p), ctypes.byref(c)
    one = {"write": lambda: lib.adaspa_cache_write(p, c, FAKE, FAKE, FAKE, None, None),
           "read": lambda: lib.adaspa_cache_read(p, c, FAKE, None, FAKE, FAKE, None),
           "attn": lambda: lib.adaspa_cache_attn(p, c, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1 << 40, None)}
    return [one[n]() if n == which else None for n in ("write", "read", "attn")]


def test_bad_pointers_are_refused(lib):
    assert _calls(lib, None, _cache()) == (1,) * 3 and _calls(lib, _prob(), None) == (1,) * 3
    for name in ("k", "v", "k_scale", "v_scale", "page_table"):
        assert _calls(lib, _prob(), _cache(**{name: None})) == (1,) * 3
        assert _calls(lib, _prob(), _cache(**{name: 0x10002})) == (1,) * 3
    p, c, odd = ctypes.byref(_prob()), ctypes.byref(_cache()), ctypes.c_void_p(0x10008)
    for bad in (None, odd):
        assert lib.adaspa_cache_write(p, c, bad, FAKE, FAKE, None, None) == 1
        assert lib.adaspa_cache_write(p, c, FAKE, bad, FAKE, None, None) == 1
        assert lib.adaspa_cache_read(p, c, FAKE, None, bad, FAKE, None) == 1
        assert lib.adaspa_cache_read(p, c, FAKE, None, FAKE, bad, None) == 1
        assert lib.adaspa_cache_attn(p, c, bad, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == 1
        assert lib.adaspa_cache_attn(p, c, FAKE, FAKE, None, bad, None, FAKE, 1 << 40, None) == 1
    two = ctypes.c_void_p(0x10002)
    for bad in (None, two):
        assert lib.adaspa_cache_write(p, c, FAKE, FAKE, bad, None, None) == 1
        assert lib.adaspa_cache_read(p, c, bad, None, FAKE, FAKE, None) == 1
        assert lib.adaspa_cache_attn(p, c, FAKE, bad, None, FAKE, None, FAKE, 1 << 40, None) == 1
    assert lib.adaspa_cache_write(p, c, FAKE, FAKE, FAKE, two, None) == 1
    assert lib.adaspa_cache_read(p, c, FAKE, two, FAKE, FAKE, None) == 1
    assert lib.adaspa_cache_attn(p, c, FAKE, FAKE, two, FAKE, None, FAKE, 1 << 40, None) == 1
    assert lib.adaspa_cache_attn(p, c, FAKE, FAKE, None, FAKE, two, FAKE, 1 << 40, None) == 1


def test_a_read_or_write_has_one_head_count(lib):
    p, c = ctypes.byref(_prob(heads=4)), ctypes.byref(_cache())
    assert lib.adaspa_cache_write(p, c, FAKE, FAKE, FAKE, None, None) == 1
    assert lib.adaspa_cache_read(p, c, FAKE, None, FAKE, FAKE, None) == 1


def test_empty_calls_need_nothing(lib):
    p, c = _prob(len=0), _Cache()
    p.pages = p.max_pages = 0
    a = ctypes.byref(p), ctypes.byref(c)
    assert lib.adaspa_cache_write(*a, None, None, None, None, None) == 0
    assert lib.adaspa_cache_read(*a, None, None, None, None, None) == 0
    assert lib.adaspa_cache_attn(*a, None, None, None, None, None, None, 0, None) == 0


def test_workspace(lib):
    """Few rows over many keys need one, and say how large; a smaller or misaligned one
    is refused."""
    p = _prob(max_pages=4096, table_stride=4096, pages=8192, len=1)
    need = lib.adaspa_cache_attn_workspace(ctypes.byref(p))
    assert need > 16 and need % 256 == 0
    args = [ctypes.byref(p), ctypes.byref(_cache()), FAKE, FAKE, None, FAKE, None]
    assert lib.adaspa_cache_attn(*args, None, need, None) == 4
    assert lib.adaspa_cache_attn(*args, FAKE, need - 1, None) == 4
    assert lib.adaspa_cache_attn(*args, ctypes.c_void_p(0x10010), need, None) == 4
    assert lib.adaspa_cache_attn_workspace(ctypes.byref(_prob(max_pages=1))) == 16
    cache = ad.KVCache(*[torch.empty(s, device="meta") for s in ((8192, 2, 16, 64), (8192, 2, 1, 64, 16), (8192, 2), (8192, 2))])
    assert ad.cache_attn_workspace((2, 2, 1, 64), cache, 4096) == need


def test_bad_shapes_are_refused_by_the_binding():
    good = ((8, 2, 32, 64), (8, 2, 2, 64, 16), (8, 2), (8, 2))
    assert _pool(*good) == good[0]
    for i, bad in ((0, (8, 2, 24, 64)), (0, (8, 2, 64)), (1, (8, 2, 32, 64)), (1, (8, 2, 2, 16, 64)), (2, (8, 3)), (3, (7, 2))):
        with pytest.raises(ad.AdaspaError):
            _pool(*good[:i], bad, *good[i + 1:])
    base = dict(pool=(8, 2, 32, 64), dtype=0, table=(2, 4), table_step=(4, 1), shape=(2, 4, 5, 64),
                strides=((1280, 320, 64, 1),), outs=None, causal=True, scale=0.0)
    _plan(*base.values())
    for kw in (dict(shape=(3, 4, 5, 64)), dict(shape=(2, 3, 5, 64)), dict(shape=(2, 4, 5, 128)), dict(table=(2,)),
               dict(table_step=(1, 2)), dict(strides=((1280, 320, 64, 2),)), dict(strides=((1280, 320, 60, 1),)),
               dict(causal=None, strides=((1280, 320, 64, 1),) * 2)):
        with pytest.raises(ad.AdaspaError):
            _plan(*dict(base, **kw).values())
    for bad in (dict(page=24), dict(head_dim=96), dict(pages=-1), dict(kv_heads=0)):
        with pytest.raises(ad.AdaspaError):
            ad.kv_cache(**dict(dict(pages=4, kv_heads=2, page=16, head_dim=64, device="meta"), **bad))


def test_tensors_elsewhere_are_refused():
    cache = ad.kv_cache(4, 2, 16, 64, device="cpu")
    t, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    for call in (lambda: ad.cache_write(x, x, cache, t, n), lambda: ad.cache_read(cache, t, n, 3),
                 lambda: ad.cache_attn(x, cache, t, n)):
        with pytest.raises(ad.AdaspaError):
            call()


def test_the_definitions():
    """Codes and roundings as torch's own conversion has them; scales by their rule."""
    code = value_of_code()
    assert torch.equal(code.nan_to_num(1e9), torch.arange(256, dtype=torch.uint8).view(E4M3).double().nan_to_num(1e9))
    g = torch.Generator().manual_seed(1)
    x = torch.cat((torch.randn(4000, generator=g) * torch.exp2(torch.randint(-12, 7, (4000,), generator=g).float()),
                   (code[:-129] + code[1:-128]).float() / 2))
    x = x[x.abs() <= 448]
    assert torch.equal(nearest(x.double()).float(), x.to(E4M3).float())
    for a, s in ((448.0, 1.0), (448.0001, 2.0), (449.0, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -126), (1.75, 2.0 ** -8),
                 (1.7578125, 2.0 ** -7), (2.9e38, 2.0 ** 119)):
        assert least_scale(torch.tensor([a, -a / 2, math.inf, math.nan], dtype=torch.float64)) == s
    # One token after another: the scale grows, older codes move with it.
    s = Sequences(1, 1, 16, 64)
    for v in (1.0, 3.3, 400.0, 5000.0):
        s.write(0, torch.full((1, 1, 64), v), torch.full((1, 1, 64), v))
    assert s.scale[0][0] == [[16.0]] and s.x[0][0][0, :, 0].tolist() == [1.0, 3.25, 384.0, 5120.0]


def test_one_place_for_keys_and_values_is_refused(lib):
    p, c = ctypes.byref(_prob(heads=2)), ctypes.byref(_cache())
    assert lib.adaspa_cache_read(p, c, FAKE, None, FAKE, FAKE, None) == 1


# Shapes of q, key heads, page, table width.  The first two in bf16: ranges of the keys without an order
# alone, with one alone.
SIZES = [((1, 24, 4096, 128), 4, 64, 64), ((1, 24, 1500, 128), 4, 64, 40), ((1, 24, 2047, 128), 4, 64, 64), ((1, 24, 2047, 128), 4, 64, 276),
         ((3, 6, 100, 64), 2, 16, 400), ((16, 24, 1, 128), 4, 64, 276), ((1, 2, 60, 64), 2, 16, 4)]


@pytest.mark.parametrize("q,Hk,page,width", SIZES)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_the_workspace_serves_the_call(lib, q, Hk, page, width, dt):
    """What is named for an order, for none, and for either is what such calls ask for."""
    B, H, L, D = q
    pages = B * width
    cache = ad.KVCache(*[torch.empty(s, device="meta") for s in
                         ((pages, Hk, page, D), (pages, Hk, page // 16, D, 16), (pages, Hk), (pages, Hk))])
    need = {}
    for causal in (True, False):
        p = _prob(batch=B, heads=H, kv_heads=Hk, len=L, head_dim=D, dtype=int(dt is torch.float16), pages=pages, page=page,
                  max_pages=width, table_stride=width, causal=int(causal), q_stride=(H * L * D, L * D, D),
                  out_stride=(H * L * D, L * D, D))
        need[causal] = lib.adaspa_cache_attn_workspace(ctypes.byref(p))
        assert need[causal] >= 16
        assert ad.cache_attn_workspace(q, cache, width, dt, causal=causal) == need[causal]
    assert ad.cache_attn_workspace(q, cache, width, dt) == max(need.values())
    if dt is torch.bfloat16 and q[2] in (4096, 1500):
        assert min(need.values()) == 16 == need[q[2] == 4096] and max(need.values()) > 16
