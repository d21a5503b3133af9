"""CPU checks of the prompt side's C ABI and binding: argument validation (no
kernel runs), bucket starts, and the 64-bit reference against differences."""
import ctypes

import pytest
import torch

import paper_2502_21079_amd as ad
from paper_2502_21079_amd.prompt import _CrossProblem, _RelBias
from _prompt_ref import bucket_index, reference, starts_by_search

FAKE = ctypes.c_void_p(0x10000)     # aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return ad.load_library()


def _prob(**kw):
    p = _CrossProblem(batch=2, heads=4, kv_heads=2, q_len=100, k_len=50, head_dim=64, dtype=0, softmax_scale=0.0)
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        L, H = (50, 2) if n in ("k", "v", "dk", "dv") else (100, 4)
        setattr(p, n + "_stride", (ctypes.c_int64 * 3)(H * L * 64, L * 64, 64))
    for k, v in kw.items():
        setattr(p, k, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return p


def _bias(**kw):
    starts = kw.pop("starts", (0, 1, 2, 3, 4, 6, 9, 13))
    arr = (ctypes.c_int32 * len(starts))(*starts)
    r = _RelBias(num_buckets=len(starts) * 2, bidirectional=1, bucket_start=ctypes.cast(
        arr, ctypes.POINTER(ctypes.c_int32)), causal=0, q_offset=0, queries_at_end=0, table_fp32=1)
    r._arr = arr
    for k, v in kw.items():
        setattr(r, k, v)
    return r


BAD = [
    (dict(batch=-1), 1), (dict(heads=0), 1), (dict(kv_heads=0), 1), (dict(kv_heads=3), 1), (dict(q_len=-1), 1),
    (dict(k_len=-1), 1), (dict(softmax_scale=float("nan")), 1), (dict(dtype=2), 2), (dict(head_dim=96), 2),
    (dict(head_dim=256), 2), (dict(batch=40000), 2), (dict(q_len=1 << 28), 2), (dict(q_stride=(1, 64, 64)), 1),
    (dict(k_stride=(-64, 64, 64)), 1), (dict(v_stride=(64, 64, 1 << 23)), 2), (dict(out_stride=(0, 6400, 64)), 1),
    (dict(out_stride=(25600, 6400, 8)), 1), (dict(key_mask_stride=-1), 1),
]


@pytest.mark.parametrize("kw,status", BAD)
def test_cross_rejects_bad_problems(lib, kw, status):
    p = _prob(**kw)
    a = [FAKE] * 3 + [None, None, FAKE, None, FAKE, 1 << 40, None]
    assert lib.adaspa_cross_attn(ctypes.byref(p), *a) == status
    assert lib.adaspa_cross_attn_workspace(ctypes.byref(p)) == 0
    a = [FAKE] * 4 + [None, None] + [FAKE] * 6 + [1 << 40, None]
    assert lib.adaspa_cross_attn_bwd(ctypes.byref(p), *a) == status
    assert lib.adaspa_cross_attn_bwd_workspace(ctypes.byref(p)) == 0


@pytest.mark.parametrize("kw,status", [(dict(dk_stride=(0, 3200, 64)), 1), (dict(dq_stride=(25600, 6400, 4)), 1),
                                       (dict(dout_stride=(25600, 6400, 1 << 24)), 2)])
def test_backward_rejects_bad_gradient_layouts(lib, kw, status):
    p = _prob(**kw)
    a = [FAKE] * 4 + [None, None] + [FAKE] * 6 + [1 << 40, None]
    assert lib.adaspa_cross_attn_bwd(ctypes.byref(p), *a) == status
    assert lib.adaspa_cross_attn_workspace(ctypes.byref(p)) > 0


def test_cross_rejects_null_and_misaligned(lib):
    p = ctypes.byref(_prob())
    good = [FAKE] * 3 + [None, None, FAKE, None, FAKE, 1 << 40, None]
    assert lib.adaspa_cross_attn(None, *good) == 1
    for i in (0, 1, 2, 5):
        for wrong in (None, ctypes.c_void_p(0x10008)):
            assert lib.adaspa_cross_attn(p, *[wrong if j == i else x for j, x in enumerate(good)]) == 1
    for i in (3, 6):
        assert lib.adaspa_cross_attn(p, *[ctypes.c_void_p(0x10002) if j == i else x for j, x in enumerate(good)]) == 1
    good = [FAKE] * 4 + [None, None] + [FAKE] * 6 + [1 << 40, None]
    for i in (0, 1, 2, 3, 6, 7, 8, 9, 10):
        assert lib.adaspa_cross_attn_bwd(p, *[None if j == i else x for j, x in enumerate(good)]) == 1


def test_workspace_checks(lib):
    p = ctypes.byref(_prob(batch=1, q_len=1, k_len=50000))
    need = lib.adaspa_cross_attn_workspace(p)
    assert need > 256 and need % 256 == 0
    a = [FAKE] * 3 + [None, None, FAKE, None]
    assert lib.adaspa_cross_attn(p, *a, None, 0, None) == 4
    assert lib.adaspa_cross_attn(p, *a, FAKE, need - 1, None) == 4
    assert lib.adaspa_cross_attn(p, *a, ctypes.c_void_p(0x10010), need, None) == 4


@pytest.mark.parametrize("kw,status", [
    (dict(num_buckets=0), 1), (dict(num_buckets=15), 1), (dict(bucket_start=None), 1), (dict(starts=(1, 2)), 1),
    (dict(starts=(0, 3, 2)), 1), (dict(starts=(0, 1025)), 2), (dict(num_buckets=514), 2), (dict(q_offset=1 << 28), 1),
    (dict(q_offset=-(1 << 28)), 1), (dict(table_fp32=2), 2)])
def test_bias_rejects_bad_buckets(lib, kw, status):
    p, r = ctypes.byref(_prob()), _bias(**kw)
    a = [FAKE] * 4 + [None, None, FAKE, None, FAKE, 1 << 40, None]
    assert lib.adaspa_rel_bias_attn(p, ctypes.byref(r), *a) == status
    assert lib.adaspa_rel_bias_attn_workspace(p, ctypes.byref(r)) == 0
    assert lib.adaspa_rel_bias_attn_bwd_workspace(p, ctypes.byref(r)) == 0
    a = [FAKE] * 5 + [None, None] + [FAKE] * 7 + [1 << 40, None]
    assert lib.adaspa_rel_bias_attn_bwd(p, ctypes.byref(r), *a) == status


def test_bias_rejects_missing_tables(lib):
    p, r = ctypes.byref(_prob()), ctypes.byref(_bias())
    a = [FAKE] * 3 + [None, None, None, FAKE, None, FAKE, 1 << 40, None]
    assert lib.adaspa_rel_bias_attn(p, r, *a) == 1
    a[3] = ctypes.c_void_p(0x10002)
    assert lib.adaspa_rel_bias_attn(p, r, *a) == 1
    assert lib.adaspa_rel_bias_attn(p, None, *[FAKE] * 4, None, None, FAKE, None, FAKE, 1 << 40, None) == 1
    a = [FAKE] * 5 + [None, None] + [FAKE] * 5 + [None, FAKE, 1 << 40, None]
    assert lib.adaspa_rel_bias_attn_bwd(p, r, *a) == 1


@pytest.mark.parametrize("n,far,both", [(32, 128, True), (32, 128, False), (8, 64, True), (64, 500, False),
                                        (4, 2, True), (2, 2, False), (16, 9, True), (320, 800, True)])
def test_bucket_starts(n, far, both):
    starts = ad.relative_bucket_starts(n, far, both)
    assert list(starts) == starts_by_search(n, far, both)
    rel = torch.arange(-2 * far, 2 * far + 1)
    at = bucket_index(rel, n, far, both)
    assert at.min() == 0 and at.max() <= n - 1
    if both:
        assert (at[rel > 0] >= n // 2).all() and (at[rel <= 0] < n // 2).all()
    else:
        assert (at[rel >= 0] == 0).all()


@pytest.mark.parametrize("n,far,both", [(1, 8, False), (2, 8, True), (7, 8, True), (32, 8, True), (0, 8, False)])
def test_bucket_starts_refuse(n, far, both):
    with pytest.raises(ad.AdaspaError):
        ad.relative_bucket_starts(n, far, both)


def test_binding_refuses_cpu_tensors():
    q = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ad.AdaspaError):
        ad.cross_attn(q, q, q)
    with pytest.raises(ad.AdaspaError):
        ad.rel_bias_attn(q, q, q, torch.zeros(32, 2))


def test_workspace_sizes_are_positive():
    assert ad.cross_attn_workspace((1, 24, 1, 128), (1, 4, 17664, 128)) > 256
    assert ad.cross_attn_bwd_workspace((1, 2, 1000, 64), (1, 2, 50, 64)) >= 256
    assert ad.rel_bias_attn_workspace((1, 2, 100, 64), (1, 2, 100, 64), 32) == 16
    assert ad.rel_bias_attn_bwd_workspace((1, 2, 1000, 64), (1, 2, 1000, 64), 32) >= 256


@pytest.mark.parametrize("both,causal,offset", [(True, False, 0), (False, True, 2), (False, True, "end")])
def test_reference_gradients_against_differences(both, causal, offset):
    """The 64-bit formulas that the kernels are held against, against central
    differences of their own forward pass: error of order step^2."""
    g = torch.Generator().manual_seed(3)
    B, H, Hk, Lq, Lk, D = 2, 4, 2, 5, 7, 8
    q, do = (torch.randn(B, H, Lq, D, generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn(B, Hk, Lk, D, generator=g, dtype=torch.float64) for _ in range(2))
    table = torch.randn(8, H, generator=g, dtype=torch.float64)
    kw = dict(key_lens=torch.tensor([7, 5]), key_mask=torch.rand(B, Lk, generator=g) > 0.2, max_distance=6,
              bidirectional=both, causal=causal, q_offset=offset, out_dtype=torch.float16)
    args = dict(q=q, k=k, v=v, table=table)
    ref = reference(q, k, v, dout=do, table=table, **kw)
    f = lambda **a: float((reference(a["q"], a["k"], a["v"], table=a["table"], **kw)["out"][0] * do).sum())  # noqa: E731
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("table", "dtable")):
        for s in range(3):
            d = torch.randn(args[name].shape, generator=g, dtype=torch.float64)
            h = 1e-5
            diff = (f(**{**args, name: args[name] + h * d}) - f(**{**args, name: args[name] - h * d})) / (2 * h)
            assert abs(diff - float((ref[grad][0] * d).sum())) <= 1e-7 * (1 + abs(diff))
