"""Attention of many rows over an 8-bit cache with every compute unit busy: several row
tiles a key head, workgroups side by side on a unit, keys that the caches answer, so that
waves drift apart.  Against the definition in 64 bits, and the same bits each time."""
import math

import pytest
import torch

import paper_2502_21079_amd as ad
from _cache_ref import SUB, U

pytestmark = pytest.mark.gpu

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def pool(B, lens, Hk, page, D, seed):
    """A pool written by the package, and what it holds, [B, Hk, n, D] in bf16."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = max(lens)
    width = -(-n // page)
    cache = ad.kv_cache(B * width + 1, Hk, page, D)
    table = torch.randperm(B * width + 1, generator=g, device=DEV)[:B * width].view(B, width).to(torch.int32)
    k = torch.randn(B, Hk, n, D, generator=g, device=DEV).to(torch.bfloat16)
    v = (torch.randn(B, Hk, n, D, generator=g, device=DEV) + 0.5).to(torch.bfloat16)
    ad.cache_write(k, v, cache, table, i32([0] * B), new_lens=i32(lens))
    return cache, table, *ad.cache_read(cache, table, i32(lens), n)


def head_reference(q, k, v, n, causal, dt):
    """(out, its bound, lse) of one head's queries, the last of n tokens, in 64 bits on the GPU.

    The bound: weights rounded to bf16 (fp16 inputs: to two bf16 values, 2^-16), sums in fp32
    (taken as 2e-5 of the sums of magnitudes), the result rounded once."""
    k, v = k[:n].double(), v[:n].double()
    s = torch.mm(q.double(), k.t().contiguous()) / math.sqrt(q.shape[1])
    if causal:
        place = n - q.shape[0] + torch.arange(q.shape[0], device=DEV)
        s.masked_fill_(torch.arange(n, device=DEV)[None] > place[:, None], -math.inf)
    z = torch.logsumexp(s, 1)
    p = torch.exp(s - z[:, None])
    out = torch.mm(p, v)
    up = 2.0 ** -8 if dt is torch.bfloat16 else 2.0 ** -16
    return out, U[dt] * out.abs() + (up + 2e-5) * torch.mm(p, v.abs()) + SUB[dt], z


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [True, False])
def test_all_units_busy(D, dt, causal):
    """272 and more row tiles: no range of the keys, then with fewer sequences some of each."""
    for B, H, Hk, Lq, lens, page in ((4, 24, 4, 720, [900, 2000, 848, 1311], 64), (1, 24, 4, 720, [3001], 16)):
        print(f"B{B} Lq{Lq} lens{lens} page{page} D{D} {dt} c{causal}", flush=True)
        cache, table, k, v = pool(B, lens, Hk, page, D, D + Lq)
        g = torch.Generator(device=DEV).manual_seed(5)
        q = torch.randn(B, Lq, H, D, generator=g, device=DEV).to(dt).transpose(1, 2)
        out, lse = ad.cache_attn(q, cache, table, i32(lens), causal=causal)
        for b in range(B):
            for h in range(H):
                ref, bound, z = head_reference(q[b, h], k[b, h * Hk // H], v[b, h * Hk // H], lens[b], causal, dt)
                over = (out[b, h].double() - ref).abs() - bound
                assert not (over > 0).any(), (b, h, float(over.max()))
                assert ((lse[b, h].double() - z).abs() <= 2e-5 * (1.0 + z.abs())).all(), (b, h)
        for _ in range(20):
            o, z = ad.cache_attn(q, cache, table, i32(lens), causal=causal)
            assert torch.equal(o, out) and torch.equal(z, lse)
