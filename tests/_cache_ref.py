"""Plain 64-bit definitions of a key/value cache in 8 bits and of attention over
it, and of rotary positions, with bounds on what a kernel may be off.

Codes: a sign, four bits of exponent (bias 7), three of fraction; all ones is no
number.  Written without torch's 8-bit types but for the storage."""
import math

import torch

E4M3 = torch.float8_e4m3fn
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SUB = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def value_of_code():
    t = []
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        x = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        t.append(math.nan if c & 127 == 127 else -x if c & 128 else x)
    return torch.tensor(t, dtype=torch.float64)


def nearest(x):
    """The nearest value with a code, ties to even; what is not finite becomes NaN."""
    fin = torch.isfinite(x)
    a = torch.where(fin, x, 0.0)
    step = torch.exp2(torch.frexp(a.abs().clamp(min=2.0 ** -6))[1].double() - 4)
    return torch.where(fin, torch.round(a / step) * step, math.nan)


def least_scale(x):
    """The least power of two s >= 2^-126 with amax <= 448 s over finite values."""
    x = x.double()
    amax = float(torch.where(torch.isfinite(x), x, 0.0).abs().max()) if x.numel() else 0.0
    e = -126
    while 448.0 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def values(cache):
    """(k, v) [pages, Hk, page, D] of a pool, in 64 bits on the CPU."""
    code = value_of_code()
    k = code[cache.k.cpu().view(torch.uint8).long()] * cache.k_scale.cpu().double()[:, :, None, None]
    v = code[cache.v.cpu().view(torch.uint8).long()] * cache.v_scale.cpu().double()[:, :, None, None, None]
    return k, v.transpose(3, 4).flatten(2, 3)


class Sequences:
    """What a cache should hold: per sequence the values, and per page and head the
    scales, written token by token as the definition has it."""

    def __init__(self, B, Hk, page, D):
        self.page, self.D, self.Hk = page, D, Hk
        self.x = [[torch.zeros(Hk, 0, D, dtype=torch.float64) for _ in range(B)] for _ in range(2)]
        self.scale = [[[] for _ in range(B)] for _ in range(2)]          # per sequence: [pages] of [Hk]

    def write(self, b, k, v):
        """k, v [Hk, n, D] behind what sequence b has."""
        for which, new in enumerate((k.cpu().double(), v.cpu().double())):
            have, scales = self.x[which][b], self.scale[which][b]
            old = have.shape[1]
            have = torch.cat((have, new), 1)
            for p in range(old // self.page, -(-have.shape[1] // self.page)):
                lo, hi = p * self.page, min((p + 1) * self.page, have.shape[1])
                row = []
                for h in range(self.Hk):
                    fresh = max(lo, old)
                    s = least_scale(have[h, fresh:hi])
                    if fresh > lo:
                        s = max(s, scales[p][h])
                    have[h, lo:hi] = nearest(have[h, lo:hi] / s) * s
                    row.append(s)
                if p < len(scales):
                    scales[p] = row
                else:
                    scales.append(row)
            self.x[which][b] = have


def attn_reference(q, ks, vs, lens, *, q_lens=None, causal=True, scale=None):
    """dict of name -> (value, bound), 64 bits; ks, vs: per sequence [Hk, n, D].

    Bounds: weights rounded to bf16 (fp16 inputs: to two bf16 values, 2^-16), sums in
    fp32 (taken as 2e-5 of the sums of magnitudes), the result rounded once."""
    B, H, Lq, D = q.shape
    u, sub = U[q.dtype], SUB[q.dtype]
    up = 2.0 ** -8 if q.dtype is torch.bfloat16 else 2.0 ** -16
    scale = scale if scale and scale > 0 else 1.0 / math.sqrt(D)
    out = torch.zeros(B, H, Lq, D, dtype=torch.float64)
    bound = torch.zeros_like(out)
    lse = torch.full((B, H, Lq), -math.inf, dtype=torch.float64)
    for b in range(B):
        k, v = ks[b].double().cpu(), vs[b].double().cpu()
        n = k.shape[1]
        G = H // k.shape[0]
        nq = Lq if q_lens is None else max(0, min(Lq, int(q_lens[b])))
        for h in range(H):
            s = (q[b, h, :nq].double().cpu() @ k[h // G].T) * scale
            if causal:
                place = n - nq + torch.arange(nq)
                s = torch.where(torch.arange(n)[None] <= place[:, None], s, -math.inf)
            z = torch.logsumexp(s, 1) if n else torch.full((nq,), -math.inf, dtype=torch.float64)
            p = torch.exp(s - torch.where(z == -math.inf, 0.0, z)[:, None])
            lse[b, h, :nq], out[b, h, :nq] = z, p @ v[h // G]
            bound[b, h, :nq] = u * out[b, h, :nq].abs() + (up + 2e-5) * (p @ v[h // G].abs()) + sub
    return {"out": (out, bound), "lse": (lse, 2e-5 * (1.0 + lse.abs()))}


def within(got, ref, what):
    """Every entry within its bound; equal infinities."""
    val, bound = ref
    g = got.double().cpu()
    assert g.shape == val.shape, f"{what}: shape {tuple(g.shape)} for {tuple(val.shape)}"
    fin = torch.isfinite(val)
    assert torch.equal(torch.isfinite(g), fin), f"{what}: finite entries differ"
    assert torch.equal(g[~fin], val[~fin]), f"{what}: infinities differ"
    over = (g - val).abs()[fin] - bound[fin]
    assert not (over > 0).any(), f"{what}: {int((over > 0).sum())} of {over.numel()} over their bound, worst by " \
                                 f"{float(over.max()):.3e}"


def random_pool(ad, B, lens, Hk, page, D, max_pages, seed, spare=3, device="cuda"):
    """A pool whose pages hold random codes and scales of powers of two (all other
    bytes NaN), a page table in no order, and the sequences' keys and values."""
    g = torch.Generator().manual_seed(seed)
    pool = B * max_pages + spare
    code = value_of_code()
    raw = [torch.randint(0, 256, (pool, Hk, page, D), generator=g, dtype=torch.uint8) for _ in range(2)]
    # Codes of magnitudes like those of numbers of unit variance against a scale of theirs.
    raw = [torch.where((r & 127) > 120, r & 0x8F, r) for r in raw]
    scale = [torch.exp2(torch.randint(-9, -4, (pool, Hk), generator=g).float()) for _ in range(2)]
    table = torch.randperm(pool, generator=g)[:B * max_pages].view(B, max_pages).to(torch.int32)
    ks, vs = [], []
    for b in range(B):
        n = lens[b]
        ids = table[b, :-(-n // page)].long()
        out = []
        for r, s in zip(raw, scale):
            x = (code[r[ids].long()] * s[ids].double()[:, :, None, None]).transpose(0, 1).reshape(Hk, len(ids) * page, D)
            out.append(x[:, :n])
            if n % page:
                r[ids[-1], :, n % page:] = 127                  # NaN behind the last token
        ks.append(out[0])
        vs.append(out[1])
    used = torch.zeros(pool, dtype=torch.bool)
    for b in range(B):
        used[table[b, :-(-lens[b] // page)].long()] = True
    for r, s in zip(raw, scale):
        r[~used] = 127
        s[~used] = math.nan
    k, v = raw
    v = v.view(pool, Hk, page // 16, 16, D).transpose(3, 4).contiguous()
    cache = ad.KVCache(k.view(E4M3).to(device), v.view(E4M3).to(device), scale[0].to(device), scale[1].to(device))
    return cache, table.to(device), ks, vs


def rotary_reference(x, freqs, *, layout="half", sections=None, magnitude=1.0, positions=None, offset=0, way=1):
    """(value, bound).  positions [B, L, axes] or None; offset: number or list [B].

    Bound: the result rounded once; sines and cosines off by 2.2e-7 (the units' own
    1.26e-7, found over 2^24 arguments, and half a step of an argument up to half a
    revolution, 2 pi 2^-26) and three fp32 roundings, 2^-21 of the magnitudes in all."""
    B, H, L, D = x.shape
    P = len(freqs)
    x = x.double().cpu()
    off = offset if isinstance(offset, (list, tuple)) else [offset] * B
    sections = sections or (P,)
    f = torch.tensor(freqs, dtype=torch.float64)
    y, bound = x.clone(), torch.zeros_like(x)
    lo = torch.arange(P) * (1 if layout == "half" else 2)
    hi = lo + (P if layout == "half" else 1)
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections))
    for b in range(B):
        pos = torch.arange(L).double()[:, None].expand(L, P) if positions is None else \
            positions[b if positions.shape[0] > 1 else 0].cpu().double()[:, axis]
        a = way * (pos + off[b]) * f
        c, s = a.cos() * magnitude, a.sin() * magnitude
        u, w = x[b][:, :, lo], x[b][:, :, hi]
        y[b][:, :, lo], y[b][:, :, hi] = u * c - w * s, u * s + w * c
        e = 2.0 ** -21 * abs(magnitude) * (u.abs() + w.abs())
        bound[b][:, :, lo], bound[b][:, :, hi] = e, e
    return y, bound
