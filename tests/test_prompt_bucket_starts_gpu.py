"""Bucket plans that only the C ABI can name, on the GPU: one bucket a direction,
whose last one begins at distance 0, and buckets that hold no distance, against the plain 64-bit form with the
gradients, at offsets where a block of scores begins on the diagonal."""
import ctypes

import pytest
import torch

import _prompt_ref
import paper_2502_21079_amd as ad
from _prompt_ref import check, reference
from paper_2502_21079_amd.prompt import _CrossProblem, _RelBias
from test_prompt_gpu import BF, HF, lens_of, make, mask_of, table_of

pytestmark = pytest.mark.gpu


def calls(q, k, v, g, table, starts, both, causal, offset, key_lens=None, key_mask=None):
    """out, lse, dq, dk, dv, dtable through the C ABI with bucket starts of the test's own."""
    lib = ad.load_library()
    (B, H, Lq, D), Hk, Lk = q.shape, k.shape[1], k.shape[2]
    p = _CrossProblem(B, H, Hk, Lq, Lk, D, 0 if q.dtype is BF else 1, 0.0)
    out, dq, dk, dv, dtable = (torch.empty_like(x) for x in (q, q, k, v, table))
    for name, x in dict(q=q, k=k, v=v, out=out, dout=g, dq=dq, dk=dk, dv=dv).items():
        setattr(p, name + "_stride", (ctypes.c_int64 * 3)(*x.stride()[:3]))
    p.key_mask_stride = Lk
    arr = (ctypes.c_int32 * len(starts))(*starts)
    r = _RelBias(len(starts) * (2 if both else 1), int(both), ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32)),
                 int(causal), 0 if offset == "end" else offset, int(offset == "end"), int(table.dtype is torch.float32))
    lse = torch.empty(B, H, Lq, device="cuda")
    p, r = ctypes.byref(p), ctypes.byref(r)
    need = max(lib.adaspa_rel_bias_attn_workspace(p, r), lib.adaspa_rel_bias_attn_bwd_workspace(p, r))
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    at = lambda x: None if x is None else x.data_ptr()  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    assert lib.adaspa_rel_bias_attn(p, r, *map(at, (q, k, v, table, key_lens, key_mask, out, lse, ws)), need, stream) == 0
    assert lib.adaspa_rel_bias_attn_bwd(p, r, *map(at, (g, q, k, v, table, key_lens, key_mask, out, lse, dq, dk, dv, dtable,
                                                        ws)), need, stream) == 0
    torch.cuda.synchronize()
    return out, lse, dq, dk, dv, dtable


def run(monkeypatch, B, H, Hk, Lq, Lk, D, dt, starts, both, causal, offset, lens="none", mask="none"):
    q, k, v, g = make(B, H, Hk, Lq, Lk, D, dt, seed=21)
    table = 2.0 * table_of(len(starts) * (2 if both else 1), H)
    kw = dict(key_lens=lens_of(B, Lk, lens), key_mask=mask_of(B, Lk, mask))
    got = calls(q, k, v, g, table, starts, both, causal, offset, **kw)
    monkeypatch.setattr(_prompt_ref, "starts_by_search", lambda *a: list(starts))
    ref = reference(q, k, v, dout=g, table=table, bidirectional=both, causal=causal, q_offset=offset, **kw)
    for name, x in zip(("out", "lse", "dq", "dk", "dv", "dtable"), got):
        check(x, ref[name], name)


@pytest.mark.parametrize("offset", [0, 1, 33, -31, "end"])
@pytest.mark.parametrize("both,causal", [(True, False), (True, True), (False, False), (False, True)])
@pytest.mark.parametrize("Lq,Lk,D", [(50, 60, 64), (50, 60, 128), (190, 223, 64), (120, 119, 128), (300, 333, 64),
                                     (300, 333, 128), (9, 1300, 64), (9, 1300, 128)])
def test_one_bucket_a_direction(Lq, Lk, D, both, causal, offset, monkeypatch):
    run(monkeypatch, 2, 2, 2, Lq, Lk, D, BF if Lq % 2 else HF, (0,), both, causal, offset)


@pytest.mark.parametrize("both", [True, False])
def test_one_bucket_a_direction_with_masks_and_shared_heads(both, monkeypatch):
    for Lq, Lk in ((70, 65), (400, 290)):
        run(monkeypatch, 3, 4, 2, Lq, Lk, 64, HF, (0, 0) if both else (0,), both, not both, 1, "empty", "some")


@pytest.mark.parametrize("both,causal", [(True, False), (False, False), (False, True)])
@pytest.mark.parametrize("starts", [(0, 0), (0, 0, 0, 5), (0, 0, 3, 3, 3, 40, 40), (0, 1, 1)])
@pytest.mark.parametrize("Lq,Lk", [(50, 60), (200, 210), (400, 500)])
def test_buckets_without_a_distance(Lq, Lk, starts, both, causal, monkeypatch):
    """Where several buckets begin at one distance the last of them holds it, and in
    one direction the keys after the query, whose distance is 0."""
    run(monkeypatch, 2, 2, 2, Lq, Lk, 64, BF, starts, both, causal, 7, "some")
