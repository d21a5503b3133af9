"""Attention over an 8-bit cache against the definition in 64 bits: rows from one to
many, lengths from none to long, pages that end inside tiles, shared heads, strides."""
import itertools
import math
import random

import pytest
import torch

import paper_2502_21079_amd as ad
from _cache_ref import attn_reference, random_pool, within

pytestmark = pytest.mark.gpu

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def queries(B, H, Lq, D, dt, seed, layout="bhld"):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(B, Lq, H, D, generator=g).to(dt).to(DEV).transpose(1, 2)
    return q if layout == "blhd" else q.contiguous()


def run(B, H, Hk, Lq, lens, page, D, dt, *, q_lens=None, causal=True, scale=None, seed=1, layout="bhld", spare=0, **kw):
    cap = max(1, -(-max(lens) // page)) + spare
    cache, table, ks, vs = random_pool(ad, B, lens, Hk, page, D, cap, seed)
    q = queries(B, H, Lq, D, dt, seed + 1, layout)
    out, lse = ad.cache_attn(q, cache, table, i32(lens), q_lens=None if q_lens is None else i32(q_lens), causal=causal,
                             scale=scale, **kw)
    ref = attn_reference(q, ks, vs, lens, q_lens=q_lens, causal=causal, scale=scale)
    what = f"B{B} H{H}/{Hk} Lq{Lq} lens{lens} page{page} D{D} {dt} q{q_lens} c{causal}"
    print(what, flush=True)
    assert out.stride() == q.stride() or not q.numel()
    within(out, ref["out"], "out " + what)
    within(lse, ref["lse"], "lse " + what)
    return q, cache, table, out, lse


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_single_tokens(page, D, dt):
    """One token of each sequence, from no key to many."""
    run(5, 4, 2, 1, [1, 0, 63, 300, 65], page, D, dt, seed=page)
    run(3, 6, 1, 1, [16, 17, 1500], page, D, dt, seed=page + 1, spare=2)


@pytest.mark.parametrize("Lq,H,Hk", [(2, 2, 2), (5, 6, 2), (16, 1, 1), (16, 2, 1), (17, 2, 1), (33, 3, 3), (128, 2, 1), (129, 1, 1),
                                     (43, 6, 2), (300, 2, 2)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_rows(Lq, H, Hk, D, causal):
    """Rows below, at and past the sizes at which a wave's or a workgroup's tiles end."""
    dt = torch.bfloat16 if (Lq + D) % 2 else torch.float16
    run(2, H, Hk, Lq, [max(Lq, 333), Lq], 32, D, dt, causal=causal, seed=Lq, layout="blhd")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_padded_batches(D, dt):
    """Samples with fewer queries than the batch is wide, with none, with more queries than
    tokens (the first see nothing), without tokens."""
    for Lq in (4, 40, 150):
        run(6, 4, 2, Lq, [200, 200, 200, 2, 0, 5], 16, D, dt, q_lens=[Lq, 1, 0, Lq, Lq, 3], seed=Lq)
        run(3, 4, 2, Lq, [200, 70, 0], 64, D, dt, q_lens=[Lq, 2, Lq], causal=False, seed=Lq + 1)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 256, 257])
def test_lengths_around_tiles(n):
    for page, Lq in ((16, 1), (128, 1), (16, 40), (64, 40)):
        run(1, 2, 1, Lq, [n], page, 64, torch.bfloat16, seed=n)


def test_large_scores_and_scales():
    """Scores of hundreds either way, scales from 2^-126 to 2^100 beside each other."""
    for Lq in (1, 70):
        run(2, 2, 1, Lq, [400, 130], 16, 64, torch.float16, scale=3.0, seed=Lq)
        run(2, 2, 1, Lq, [400, 130], 16, 128, torch.bfloat16, scale=-1.0, seed=Lq + 1)
        for dt in (torch.bfloat16, torch.float16):
            B, H, page, D, lens = 1, 2, 16, 64, [200]
            cache, table, ks, vs = random_pool(ad, B, lens, 1, page, D, 13, Lq)
            ids = table[0].long().cpu()
            by = torch.ones(13, dtype=torch.float64)
            # One page of values thousands of times larger whose keys hardly count, one of zeros of the least scale.
            by[2], by[5] = 2.0 ** 10, 2.0 ** -117
            at = torch.arange(200) // page
            cache.v_scale[ids.to(DEV)] *= by.float().to(DEV)[:, None]
            vs[0] = vs[0] * by[at][None, :, None]
            ks[0][:, at == 2] = 0
            cache.k[ids[2].item()] = torch.zeros_like(cache.k[ids[2].item()].float()).to(cache.k.dtype)
            q = queries(B, H, Lq, D, dt, 9) * 4
            out, lse = ad.cache_attn(q, cache, table, i32(lens))
            ref = attn_reference(q, ks, vs, lens)
            within(out, ref["out"], "out")
            within(lse, ref["lse"], "lse")


def test_pages_that_are_not_there():
    """Entries outside the pool take no part, nor do their tokens' places."""
    B, H, Hk, page, D = 1, 4, 2, 16, 64
    for Lq in (1, 50):
        lens = [200]
        cache, table, ks, vs = random_pool(ad, B, lens, Hk, page, D, 13, 3)
        q = queries(B, H, Lq, D, torch.bfloat16, 4)
        bad = table.clone()
        bad[0, 1], bad[0, 6], bad[0, 7] = -1, cache.k.shape[0], 1 << 30
        keep = torch.ones(200, dtype=torch.bool)
        keep[16:32] = keep[96:128] = False
        out, lse = ad.cache_attn(q, cache, bad, i32(lens), causal=False)
        ref = attn_reference(q, [ks[0][:, keep]], [vs[0][:, keep]], [int(keep.sum())], causal=False)
        within(out, ref["out"], "out")
        within(lse, ref["lse"], "lse")
        out, lse = ad.cache_attn(q, cache, torch.full_like(bad, -1), i32(lens))
        assert not out.any() and (lse == -math.inf).all()
        # Lengths past the table end with it, below 0 count as 0.
        full = [13 * page]
        cache, table, ks, vs = random_pool(ad, B, full, Hk, page, D, 13, 5)
        out, lse = ad.cache_attn(q, cache, table, i32([1 << 30]))
        ref = attn_reference(q, ks, vs, full)
        within(out, ref["out"], "out")
        out, lse = ad.cache_attn(q, cache, table, i32([-4]))
        assert not out.any() and (lse == -math.inf).all()
        none = table[:, :0]
        out, lse = ad.cache_attn(q, cache, none, i32([10]))
        assert not out.any() and (lse == -math.inf).all()


def test_nan_of_a_token_reaches_its_rows_alone():
    """A sequence with a NaN among its keys, or values, gives NaN there; others do not."""
    for Lq in (1, 60):
        cache, table, ks, vs = random_pool(ad, 2, [100, 100], 1, 16, 64, 7, 8)
        q = queries(2, 2, Lq, 64, torch.bfloat16, 9)
        cache.k.view(torch.uint8)[table[0, 2].long(), 0, 3, 5] = 0x7F
        out, lse = ad.cache_attn(q, cache, table, i32([100, 100]))
        assert out[0].isnan().all() and lse[0].isnan().all()
        ref = attn_reference(q[1:], ks[1:], vs[1:], [100])
        within(out[1:], ref["out"], "out")
        within(lse[1:], ref["lse"], "lse")


def test_outputs_workspace_and_repeats():
    """Outputs and workspace of the caller's; the same bits each time, whatever the workspace
    held; no lse; one device call per stream."""
    B, H, Hk, page, D = 3, 8, 2, 64, 128
    lens = [900, 1200, 64]
    cache, table, ks, vs = random_pool(ad, B, lens, Hk, page, D, 19, 6)
    for Lq in (1, 4, 30):
        q = queries(B, H, Lq, D, torch.bfloat16, Lq, "blhd")
        out, lse = ad.cache_attn(q, cache, table, i32(lens))
        need = ad.cache_attn_workspace(q.shape, cache, 19)
        for byte in (0, 255):
            ws = torch.full((need,), byte, dtype=torch.uint8, device=DEV)
            room = torch.full((B, Lq + 1, H + 1, D), 3.0, dtype=q.dtype, device=DEV)
            o = room[:, :Lq, :H].transpose(1, 2)
            z = torch.empty_like(lse)
            ad.cache_attn(q, cache, table, i32(lens), out=o, lse=z, workspace=ws)
            assert torch.equal(o, out) and torch.equal(z, lse)
            assert (room[:, Lq:] == 3).all() and (room[:, :, H:] == 3).all()
        o, none = ad.cache_attn(q, cache, table, i32(lens), want_lse=False)
        assert none is None and torch.equal(o, out)
        if need > 16:
            with pytest.raises(ad.AdaspaError):
                ad.cache_attn(q, cache, table, i32(lens), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            o, z = ad.cache_attn(q, cache, table, i32(lens))
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(o, out) and torch.equal(z, lse)


def test_shared_pages():
    """Two sequences over the same beginning, read alike."""
    cache, table, ks, vs = random_pool(ad, 1, [256], 2, 32, 64, 8, 7)
    both = table.expand(2, -1)                           # a table of one row, read twice
    q = queries(2, 4, 3, 64, torch.bfloat16, 1)
    out, lse = ad.cache_attn(q, cache, both, i32([256, 100]))
    ref = attn_reference(q, [ks[0], ks[0][:, :100]], [vs[0], vs[0][:, :100]], [256, 100])
    within(out, ref["out"], "out")
    within(lse, ref["lse"], "lse")


def test_long_sequences():
    """Tens of thousands of tokens, split over workgroups, in both kernels."""
    run(2, 4, 1, 1, [20011, 9000], 64, 64, torch.bfloat16, seed=1)
    run(1, 6, 2, 3, [30000], 16, 128, torch.float16, seed=2)
    run(1, 2, 1, 130, [12345], 128, 128, torch.bfloat16, seed=3)


def test_random_cases():
    rng = random.Random(11)
    for trial in range(60):
        page, D, dt = rng.choice([16, 32, 64, 128]), rng.choice([64, 128]), rng.choice([torch.bfloat16, torch.float16])
        Hk, G, B = rng.choice([1, 2, 3]), rng.choice([1, 2, 3, 5, 8, 12]), rng.choice([1, 2, 4])
        Lq = rng.choice([1, 1, 2, 3, 7, 20, 65, 140])
        lens = [rng.choice([0, 1, rng.randrange(700)]) for _ in range(B)]
        q_lens = [rng.randrange(-1, Lq + 2) for _ in range(B)] if rng.random() < 0.5 else None
        run(B, Hk * G, Hk, Lq, lens, page, D, dt, q_lens=q_lens, causal=rng.random() < 0.7, seed=trial,
            layout=rng.choice(["bhld", "blhd"]), spare=rng.randrange(20), scale=rng.choice([None, 0.3]))


def test_sizes_of_nothing():
    for B, Lq in itertools.product((0, 2), (0, 1)):
        if B and Lq:
            continue
        cache = ad.kv_cache(4, 2, 16, 64)
        q = torch.zeros(B, 4, Lq, 64, dtype=torch.bfloat16, device=DEV)
        out, lse = ad.cache_attn(q, cache, torch.zeros(B, 3, dtype=torch.int32, device=DEV),
                                 torch.zeros(B, dtype=torch.int32, device=DEV))
        assert out.shape == q.shape and lse.shape == q.shape[:3]


def long_pool(B, lens, Hk, page, D, seed, max_pages):
    """A pool made on the GPU: unit-variance keys, values with a mean, and the sequences'
    keys and values on the CPU in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    pool = B * max_pages + 2
    cache = ad.kv_cache(pool, Hk, page, D)
    table = torch.randperm(pool, generator=g, device=DEV)[:B * max_pages].view(B, max_pages).to(torch.int32)
    n = max(lens)
    k = torch.randn(B, Hk, n, D, generator=g, device=DEV).to(torch.bfloat16)
    v = (torch.randn(B, Hk, n, D, generator=g, device=DEV) + 0.5).to(torch.bfloat16)
    ad.cache_write(k, v, cache, table, i32([0] * B), new_lens=i32(lens))
    k, v = ad.cache_read(cache, table, i32(lens), n)
    return cache, table, [k[b, :, :lens[b]] for b in range(B)], [v[b, :, :lens[b]] for b in range(B)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_over_many_tiles(D, dt, causal):
    """Walks of more than 64 tiles (page numbers are read 64 at a time), ranges that end inside
    a sequence, rows that fill the last tile in part."""
    for B, H, Hk, Lq, lens, page in ((2, 3, 1, 100, [9000, 4200], 16), (1, 2, 2, 700, [5003], 128)):
        cache, table, ks, vs = long_pool(B, lens, Hk, page, D, Lq + D, -(-max(lens) // page))
        q = queries(B, H, Lq, D, dt, 3, "blhd")
        out, lse = ad.cache_attn(q, cache, table, i32(lens), causal=causal)
        ref = attn_reference(q, ks, vs, lens, causal=causal)
        within(out, ref["out"], "out")
        within(lse, ref["lse"], "lse")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_late_keys_far_above_the_first(dt):
    """Rows whose reference is set by small scores, then meet ones above it by 10, 40 and 120
    powers of two: moved, or worked on again."""
    for Lq in (1, 20, 90):
        for above in (10.0, 40.0, 120.0):
            cache, table, ks, vs = long_pool(1, [1500], 1, 64, 64, 5, 24)
            q = queries(1, 2, Lq, 64, dt, 6)
            q[..., 0] = 1.0
            k = ks[0].clone()
            k[..., 0] = 0
            k[:, 700, 0] = above * math.log(2.0) * 8.0        # one key: the score is that over sqrt(64)
            cache = ad.kv_cache(26, 1, 64, 64)
            ad.cache_write(k[None], vs[0][None], cache, table, i32([0]))
            k, v = ad.cache_read(cache, table, i32([1500]), 1500)
            out, lse = ad.cache_attn(q, cache, table, i32([1500]), causal=False)
            ref = attn_reference(q, [k[0]], [v[0]], [1500], causal=False)
            within(out, ref["out"], f"out {Lq} {above}")
            within(lse, ref["lse"], f"lse {Lq} {above}")


def test_queries_behind_the_last_may_be_anything():
    """Padding queries of NaN and infinity change no other row's bits."""
    for Lq in (4, 30, 200):
        cache, table, ks, vs = long_pool(2, [900, 700], 2, 32, 64, 7, 29)
        q = queries(2, 4, Lq, 64, torch.bfloat16, 8)
        n = [Lq, Lq // 2]
        out, lse = ad.cache_attn(q, cache, table, i32([900, 700]), q_lens=i32(n))
        q[1, :, n[1]:] = math.nan
        q[1, :, n[1]::2] = math.inf
        out2, lse2 = ad.cache_attn(q, cache, table, i32([900, 700]), q_lens=i32(n))
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        assert not out[1, :, n[1]:].any() and (lse[1, :, n[1]:] == -math.inf).all()


def test_an_empty_pool_and_many_samples():
    """No page at all; several hundred samples, most of them empty; a table far wider than the
    sequences are long."""
    cache = ad.kv_cache(0, 2, 16, 64)
    for Lq in (1, 70):
        q = queries(3, 4, Lq, 64, torch.bfloat16, 1)
        out, lse = ad.cache_attn(q, cache, torch.zeros(3, 300, dtype=torch.int32, device=DEV), i32([4000, 1, 0]))
        assert not out.any() and (lse == -math.inf).all()
    rng = random.Random(3)
    lens = [rng.choice([0, 0, 0, rng.randrange(90)]) for _ in range(600)]
    cache, table, ks, vs = random_pool(ad, 600, lens, 1, 16, 64, 6, 2, spare=0)
    wide = torch.full((600, 200), -1, dtype=torch.int32, device=DEV)
    wide[:, :6] = table
    for Lq, q_lens in ((1, None), (3, [rng.randrange(4) for _ in range(600)])):
        q = queries(600, 2, Lq, 64, torch.bfloat16, 3)
        out, lse = ad.cache_attn(q, cache, wide, i32(lens), q_lens=None if q_lens is None else i32(q_lens))
        ref = attn_reference(q, ks, vs, lens, q_lens=q_lens)
        within(out, ref["out"], "out")
        within(lse, ref["lse"], "lse")


def test_rows_without_a_token_are_zeros_beside_tokens_that_are_no_numbers():
    """Padding queries, and queries that stand before the first token, where values of the
    sequence are NaN; a row that stands before those in another range of the keys than theirs."""
    for Lq, n in ((3, 300), (3, 5000), (40, 300), (40, 9000), (150, 9000)):
        cache, table, ks, vs = random_pool(ad, 2, [n, 2], 2, 64, 64, -(-n // 64), Lq)
        q = queries(2, 4, Lq, 64, torch.bfloat16, 4)
        nq = [Lq // 2, Lq]                                # the second sample's first queries see nothing
        for t in (5, n // 2):
            cache.k[table[0, t // 64].long(), :, t % 64] = math.nan
            cache.v[table[0, t // 64].long(), :, t % 64 // 16, :, t % 16] = math.nan
        cache.v[table[1, 0].long(), :, 0, :, 1] = math.nan
        out, lse = ad.cache_attn(q, cache, table, i32([n, 2]), q_lens=i32(nq))
        assert not out[0, :, nq[0]:].any() and (lse[0, :, nq[0]:] == -math.inf).all()
        assert torch.isnan(out[0, :, :nq[0]]).all()
        assert not out[1, :, :Lq - 2].any() and (lse[1, :, :Lq - 2] == -math.inf).all()


@pytest.mark.parametrize("Lq,H,Hk", [(33, 1, 1), (16, 6, 2), (17, 4, 2), (48, 2, 2), (49, 1, 1), (8, 6, 1), (12, 4, 1)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_rows_around_48_over_long_sequences(Lq, H, Hk, D, dt):
    for causal, q_lens in ((True, None), (False, None), (True, [Lq, 0, Lq - 5, Lq, 1])):
        run(5, H, Hk, Lq, [3100, 300, 17, 0, 2900], 32, D, dt, causal=causal, q_lens=q_lens, seed=Lq, layout="blhd")


def test_pages_past_4_gb():
    """Pages all over a pool of more than 4 GB give what the same pages give side by side."""
    page, Hk, D, width = 128, 8, 128, 25
    pages = (1 << 32) // (page * Hk * D) + 40
    g = torch.Generator(device=DEV).manual_seed(1)
    n = page * width - 5
    k, v = (torch.randn(1, Hk, n, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    far, near = ad.kv_cache(pages, Hk, page, D), ad.kv_cache(width, Hk, page, D)
    spread = i32([[pages - 1 - i * (pages // width) for i in range(width)]])
    side = torch.arange(width, dtype=torch.int32, device=DEV)[None]
    ad.cache_write(k, v, far, spread, i32([0]))
    ad.cache_write(k, v, near, side, i32([0]))
    for Lq in (1, 20, 40, 60):
        q = queries(1, Hk, Lq, D, torch.bfloat16, Lq)
        for a, b in zip(ad.cache_attn(q, far, spread, i32([n])), ad.cache_attn(q, near, side, i32([n]))):
            assert torch.equal(a, b) and torch.isfinite(a).all()


@pytest.mark.parametrize("causal", [True, False, None])
def test_a_workspace_of_the_size_named(causal):
    """Exactly as many bytes as are named, at shapes where an order and none want different
    amounts; the bits are those of a call that allocates its own."""
    for B, H, Hk, Lq, n, D, page in ((1, 24, 4, 4096, 4096, 128, 64), (1, 24, 4, 1500, 2500, 128, 64),
                                     (2, 6, 2, 300, 400, 64, 16)):
        width = -(-n // page)
        cache, table, ks, vs = long_pool(B, [n] * B, Hk, page, D, 3, width)
        q = queries(B, H, Lq, D, torch.bfloat16, 4)
        ws = torch.empty(ad.cache_attn_workspace(q.shape, cache, width, causal=causal), dtype=torch.uint8, device=DEV)
        for order in (True, False) if causal is None else (causal,):
            ws.fill_(255)
            got = ad.cache_attn(q, cache, table, i32([n] * B), causal=order, workspace=ws)
            want = ad.cache_attn(q, cache, table, i32([n] * B), causal=order)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("H,Hk,Lq,lens", [(2, 2, 1, [300, 1984, 40]), (12, 2, 1, [9000, 5]), (8, 1, 3, [4000, 700]),
                                          (6, 1, 7, [5000, 3100]), (3, 3, 9, [130, 64])])
@pytest.mark.parametrize("D", [64, 128])
def test_few_rows_lose_no_bits_to_their_weights(H, Hk, Lq, lens, D):
    """bf16 with up to 48 rows a key head: weights are two bf16 values, so what remains of them is
    2^-16, as with fp16, and the result's own rounding (2^-8) is all of its size."""
    cache, table, ks, vs = random_pool(ad, len(lens), lens, Hk, 32, D, -(-max(lens) // 32), Lq + D)
    q = queries(len(lens), H, Lq, D, torch.bfloat16, Lq)
    out, lse = ad.cache_attn(q, cache, table, i32(lens))
    want, abs_sum = (attn_reference(q, ks, [f(v) for v in vs], lens)["out"][0] for f in (lambda v: v, torch.abs))
    within(out, (want, 2.0 ** -8 * want.abs() + (2.0 ** -16 + 2e-5) * abs_sum), "out")
