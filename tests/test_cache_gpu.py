"""Quantising a cache as it is written, and reading it back, against the definition
in 64 bits, bit for bit."""
import math
import random

import pytest
import torch

import paper_2502_21079_amd as ad
from _cache_ref import E4M3, Sequences, random_pool, values

pytestmark = pytest.mark.gpu

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def fresh_cache(pages, Hk, page, D, fill=0x7F):
    """A pool of NaN (or another byte) with scales of NaN."""
    c = ad.kv_cache(pages, Hk, page, D)
    for t in (c.k, c.v):
        t.view(torch.uint8).fill_(fill)
    c.k_scale.fill_(math.nan)
    c.v_scale.fill_(math.nan)
    return c


def tokens(B, Hk, T, D, dt, seed, layout="bhld", spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, T, Hk, D, generator=g) * torch.exp(spread * torch.randn(B, T, Hk, 1, generator=g))
    x = x.clamp(-6e4, 6e4).to(dt).to(DEV).transpose(1, 2)
    return x if layout == "blhd" else x.contiguous()


def raw(cache):
    """The pool's bytes: codes and the scales' bits (NaN among them)."""
    return cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale.view(torch.int32), \
        cache.v_scale.view(torch.int32)


def expect(cache, table, seqs, lens):
    """Codes and scales of the pool are those of the definition, for the tokens that are
    there."""
    got, scales = values(cache), (cache.k_scale.cpu().double(), cache.v_scale.cpu().double())
    page = seqs.page
    for which in range(2):
        for b, n in enumerate(lens):
            want = seqs.x[which][b]
            assert want.shape[1] == n
            ids = table[b, :-(-n // page)].cpu().long()
            for p, i in enumerate(ids):
                assert scales[which][i].tolist() == seqs.scale[which][b][p], (which, b, p)
            x = got[which][ids].transpose(0, 1).reshape(want.shape[0], len(ids) * page, -1)[:, :n]
            assert torch.equal(x.nan_to_num(1e30), want.nan_to_num(1e30)), (which, b)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_prompts_then_tokens(page, D, dt):
    """A ragged prompt, a second piece that begins inside pages, then single tokens, one of
    which makes a scale grow."""
    B, Hk, most = 3, 2, 260
    cap = -(-most // page)
    g = torch.Generator().manual_seed(page + D)
    table = torch.randperm(B * cap + 2, generator=g)[:B * cap].view(B, cap).to(torch.int32).to(DEV)
    cache = fresh_cache(B * cap + 2, Hk, page, D)
    seqs, lens = Sequences(B, Hk, page, D), [0] * B
    steps = [(133, [133, 1, 70], "blhd"), (35, [35, 35, 0], "bhld")] + [(1, None, "bhld")] * 4
    for i, (T, new, layout) in enumerate(steps):
        k, v = tokens(B, Hk, T, D, dt, 10 * i + 1, layout), tokens(B, Hk, T, D, dt, 10 * i + 2, layout)
        if i == 4:
            k[:, 1], v[0] = 3.0e4, -2.5e4
        ad.cache_write(k, v, cache, table, i32(lens), new_lens=None if new is None else i32(new))
        for b in range(B):
            n = T if new is None else new[b]
            seqs.write(b, k[b, :, :n], v[b, :, :n])
            lens[b] += n
        expect(cache, table, seqs, lens)
    # Read back, whole and from odd places on; rows that are no token's are zeros.
    for dtype in (torch.bfloat16, torch.float16):
        for starts, T in ((None, 200), ([0, 5, 17], 50), ([150, -3, 40], 33), ([100, 20, 90], 1)):
            k, v = ad.cache_read(cache, table, i32(lens), T, starts=None if starts is None else i32(starts), dtype=dtype)
            for which, x in enumerate((k, v)):
                for b in range(B):
                    s = 0 if starts is None else starts[b]
                    want = torch.zeros(Hk, T, D, dtype=torch.float64)
                    lo, hi = max(s, 0), min(s + T, lens[b])
                    if hi > lo:
                        want[:, lo - s:hi - s] = seqs.x[which][b][:, lo:hi]
                    assert torch.equal(x[b].cpu(), want.to(dtype)), (which, b, starts)


@pytest.mark.parametrize("page", [16, 64])
def test_what_was_there_stays(page):
    """Bytes behind the last token, pages of no sequence and pages that the table names
    wrongly are left as they were."""
    B, Hk, D, T = 2, 2, 64, 21
    cache = fresh_cache(8, Hk, page, D, fill=0x55)
    cache.k_scale.fill_(7.0)
    before = [t.clone() for t in raw(cache)]
    table = i32([[3, 1, 9, 9], [-1, 8, 1 << 30, -5]])        # the second sequence has no page at all
    k, v = tokens(B, Hk, T, D, torch.bfloat16, 1), tokens(B, Hk, T, D, torch.bfloat16, 2)
    ad.cache_write(k, v, cache, table, i32([0, 0]))
    used = [3, 1][:-(-T // page)]
    others = [p for p in range(8) if p not in used]
    for t, was in zip(raw(cache), before):
        assert torch.equal(t[others], was[others])
    tail = T - (len(used) - 1) * page
    assert (cache.k.view(torch.uint8)[used[-1], :, tail:] == 0x55).all()
    rows = cache.v.view(torch.uint8)[used[-1]].transpose(2, 3).reshape(Hk, page, D)
    assert (rows[:, tail:] == 0x55).all() and not (rows[:, :tail] == 0x55).all()
    # Lengths below 0 and behind the table's end write nothing; zeros are read there.
    now = [t.clone() for t in raw(cache)]
    for lens, new in (([-1, -5], None), ([4 * page, 1 << 30], None), ([5, 5], [0, -7]), ([(1 << 31) - 1] * 2, None)):
        ad.cache_write(k, v, cache, table, i32(lens), new_lens=None if new is None else i32(new))
    for t, was in zip(raw(cache), now):
        assert torch.equal(t, was)
    for lens in ([-3, 40], [0, 1 << 30]):
        a, b = ad.cache_read(cache, table, i32(lens), 60)
        assert not a.any() and not b.any()
    a, b = ad.cache_read(cache, table, i32([1 << 30, 1 << 30]), 10, starts=i32([(1 << 31) - 4, -(1 << 31)]))
    assert not a.any() and not b.any()
    # Outputs of the caller's, in place of a wider tensor; nothing beside them is written.
    room = torch.full((B, 25, 3, D), 9.0, dtype=torch.bfloat16, device=DEV)
    out = room[:, :T, :2].transpose(1, 2)
    a, b = ad.cache_read(cache, table, i32([T, T]), T, k=out)
    assert a.data_ptr() == out.data_ptr() and (room[:, T:] == 9).all() and (room[:, :, 2] == 9).all()
    c, _ = ad.cache_read(cache, table, i32([T, T]), T)
    assert torch.equal(out, c) and not out[1].any()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
def test_extreme_values(dt):
    """Zeros, the type's largest and least values, infinities and NaN."""
    Hk, page, D = 3, 16, 64
    big, tiny = torch.finfo(dt).max, torch.finfo(dt).tiny
    k = torch.zeros(1, Hk, 32, D, dtype=dt, device=DEV)
    k[0, 0, 0, :8] = torch.tensor([big, -big / 2, 1.0, tiny, -0.0, big / 500, -1.0, 3.0], dtype=dt)
    k[0, 1, :4, 0] = torch.tensor([math.inf, -math.inf, math.nan, 1.0], dtype=dt)
    k[0, 1, 5] = tokens(1, 1, 1, D, dt, 3)[0, 0, 0]
    k[0, 2, 0, :4] = torch.tensor([tiny, tiny / 4, -tiny, tiny * 448], dtype=dt)
    k[0, 2, 20] = math.nan                               # a page with nothing finite but zeros
    v = k.flip(3).contiguous()
    cache, table = fresh_cache(2, Hk, page, D), i32([[1, 0]])
    seqs = Sequences(1, Hk, page, D)
    ad.cache_write(k, v, cache, table, i32([0]))
    seqs.write(0, k[0], v[0])
    expect(cache, table, seqs, [32])
    a, b = ad.cache_read(cache, table, i32([32]), 32)
    for x, want in ((a, seqs.x[0][0]), (b, seqs.x[1][0])):
        assert torch.equal(x[0].cpu().nan_to_num(1.5, 1e38), want.float().to(torch.bfloat16).nan_to_num(1.5, 1e38))
    # A larger token behind them moves zeros, subnormal codes and NaN along.
    more = torch.full((1, Hk, 1, D), 7.0, dtype=dt, device=DEV)
    ad.cache_write(more, more, cache, table, i32([9]))
    seqs2 = Sequences(1, Hk, page, D)
    seqs2.write(0, k[0, :, :16], v[0, :, :16])
    for w in range(2):
        seqs2.x[w][0] = seqs2.x[w][0][:, :9]
    seqs2.write(0, more[0], more[0])
    got = values(cache)
    for w in range(2):
        assert torch.equal(got[w][1][:, :10].nan_to_num(1e30), seqs2.x[w][0].nan_to_num(1e30))
        assert (cache.k_scale, cache.v_scale)[w][1].tolist() == seqs2.scale[w][0][0]


def test_many_sizes():
    """Random shapes, layouts, places and lengths against the definition."""
    rng = random.Random(5)
    for trial in range(25):
        page, D, dt = rng.choice([16, 32, 64, 128]), rng.choice([64, 128]), rng.choice([torch.bfloat16, torch.float16])
        B, Hk, T = rng.choice([1, 2, 5]), rng.choice([1, 2, 3]), rng.choice([1, 2, 15, 16, 17, 63, 64, 65, 127, 200])
        lens = [rng.randrange(0, 150) for _ in range(B)]
        new = [rng.randrange(0, T + 1) for _ in range(B)] if rng.random() < 0.5 else [T] * B
        cap = -(-max(n + m for n, m in zip(lens, new)) // page) + rng.randrange(2)
        g = torch.Generator().manual_seed(trial)
        table = torch.randperm(B * cap + 1, generator=g)[:B * cap].view(B, cap).to(torch.int32).to(DEV)
        cache, seqs = fresh_cache(B * cap + 1, Hk, page, D), Sequences(B, Hk, page, D)
        at = [0] * B
        for width, counts in ((max(lens), lens), (T, new)):
            k = tokens(B, Hk, width, D, dt, trial * 7 + width, rng.choice(["bhld", "blhd"]), 1.0)
            v = tokens(B, Hk, width, D, dt, trial * 7 + width + 1, rng.choice(["bhld", "blhd"]), 1.0)
            ad.cache_write(k, v, cache, table, i32(at), new_lens=i32(counts))
            for b in range(B):
                seqs.write(b, k[b, :, :counts[b]], v[b, :, :counts[b]])
                at[b] += counts[b]
        expect(cache, table, seqs, at)


def test_long_offsets():
    """Pages past 4 GB of a pool, written and read at the far end."""
    page, Hk, D = 128, 8, 128
    pages = (1 << 32) // (page * Hk * D) + 40
    cache = ad.kv_cache(pages, Hk, page, D)
    table = i32([[0, pages - 1, pages // 2, pages - 3]])
    k, v = tokens(1, Hk, 400, D, torch.bfloat16, 1), tokens(1, Hk, 400, D, torch.bfloat16, 2)
    ad.cache_write(k, v, cache, table, i32([0]))
    seqs = Sequences(1, Hk, page, D)
    seqs.write(0, k[0], v[0])
    a, b = ad.cache_read(cache, table, i32([400]), 400)
    assert torch.equal(a[0].cpu().double(), seqs.x[0][0]) and torch.equal(b[0].cpu().double(), seqs.x[1][0])
    q = tokens(1, Hk, 1, D, torch.bfloat16, 3, spread=0.0)
    far, _ = ad.cache_attn(q, cache, table, i32([400]))
    small = ad.kv_cache(4, Hk, page, D)
    ad.cache_write(k, v, small, i32([[0, 1, 2, 3]]), i32([0]))
    near, _ = ad.cache_attn(q, small, i32([[0, 1, 2, 3]]), i32([400]))
    assert torch.equal(far, near)


def test_a_pool_that_was_not_written_here():
    """Reading takes codes, scales, table and lengths as they are."""
    cache, table, ks, vs = random_pool(ad, 3, [77, 0, 130], 2, 32, 128, 5, seed=4)
    k, v = ad.cache_read(cache, table, i32([77, 0, 130]), 160)
    for b, n in enumerate((77, 0, 130)):
        assert torch.equal(k[b, :, :n].cpu().double(), ks[b]) and torch.equal(v[b, :, :n].cpu().double(), vs[b])
        assert not k[b, :, n:].any() and not v[b, :, n:].any()
    assert cache.k.dtype is E4M3


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_idle_samples_write_nothing(page, D):
    """Samples without new tokens, whose lengths end inside a page: it stays as it was, bit for
    bit, also where another sequence writes it and its scale grows."""
    Hk, T, idle = 3, 5, 200
    cache = fresh_cache(4, Hk, page, D)
    k, v = tokens(2, Hk, T, D, torch.bfloat16, 1), tokens(2, Hk, T, D, torch.bfloat16, 2)
    before = [t.clone() for t in raw(cache)]
    ad.cache_write(k, v, cache, i32([[1, 2], [3, 0]]), i32([7, page + 3]), new_lens=i32([0, -4]))
    for t, was in zip(raw(cache), before):
        assert torch.equal(t, was)
    # One sequence in use among many slots that still name its page.
    table = torch.ones(idle + 1, 1, dtype=torch.int32, device=DEV)
    seqs, lens, new = Sequences(1, Hk, page, D), [3] * (idle + 1), [0] * (idle + 1)
    g = torch.Generator().manual_seed(3)
    for step, n in enumerate((3, 1, 1, 1, 1, 1, 1, 1)):
        k, v = (torch.randn(1, Hk, T, D, generator=g).to(torch.bfloat16) * 4 ** step for _ in range(2))
        k, v = k.to(DEV), v.to(DEV)
        lens[idle // 2], new[idle // 2] = (2 + step if step else 0), n
        ad.cache_write(k.expand(idle + 1, -1, -1, -1), v.expand(idle + 1, -1, -1, -1), cache, table, i32(lens),
                       new_lens=i32(new))
        seqs.write(0, k[0, :, :n], v[0, :, :n])
        expect(cache, table[:1], seqs, [3 + step])
