"""Performance cases of the prompt side of a video diffusion transformer: cross
attention to an encoder's states, and attention with a learned relative
position bias by buckets, each forward and as a training step.

Kinds:

* ``cross``        :func:`cross_attn`: queries of one length, keys and values
                   of another (an encoder's states);
* ``cross_train``  the same with its backward pass: the output and the
                   gradients of q, k and v;
* ``bias``         :func:`rel_bias_attn`: scores plus a learned value per
                   bucket of the distance between key and query;
* ``bias_train``   the same with its backward pass, the table's gradient among
                   the outputs.

Lengths and heads are those of the package's workloads (a preview of 1,984
video tokens with 64 text tokens, a clip of 17,664 with 256, a long video of
110,080 with 256) or lie between them.
"""
import math

import torch

own = False

DEV = "cuda"


def _case(name, kind, batch, heads, q_len, k_len, head_dim, dtype="bf16", kv_heads=0, layout="bhld", ragged=False,
          empty=False, mask=False, buckets=0, max_distance=0, both_ways=True, causal=False, at_end=False, scale=0.0):
    c = dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads or heads, q_len=q_len, k_len=k_len,
             head_dim=head_dim, dtype=dtype, layout=layout, ragged=ragged, empty=empty, mask=mask, buckets=buckets,
             max_distance=max_distance, both_ways=both_ways, causal=causal, at_end=at_end, scale=scale)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # Video tokens read the prompt's states: the smallest preview; the
        # moderate clip, guided and unguided side by side with prompts of
        # different lengths, heads as the projection left them; the long video.
        _case("cross_preview", "cross", 1, 2, 1984, 64, 64),
        _case("cross_moderate_pair", "cross", 2, 48, 17664, 256, 64, layout="blhd", ragged=True),
        _case("cross_long", "cross", 1, 24, 110080, 256, 128),
        # The other direction: one pooling query per sample over a clip's
        # states, key heads shared by six query heads; a prompt's 256 tokens
        # reading the long video.
        _case("cross_one_query", "cross", 4, 24, 1, 17664, 128, dtype="fp16", kv_heads=4),
        _case("cross_text_reads_video", "cross", 1, 24, 256, 110080, 128),
        # Training: a short clip of odd length, three samples of which one has
        # its prompt dropped, single states masked; and the long video.
        _case("cross_train_ragged", "cross_train", 3, 12, 4999, 226, 64, dtype="fp16", layout="blhd", ragged=True,
              empty=True, mask=True),
        _case("cross_train_long", "cross_train", 1, 24, 110080, 256, 128),
        # The text encoder's own attention: two prompts; a document of odd
        # length; one new token per sequence in a decoder with a cache.
        _case("bias_prompt", "bias", 2, 24, 256, 256, 64, ragged=True, buckets=32, max_distance=128, scale=1.0),
        _case("bias_document", "bias", 1, 12, 8191, 8191, 64, buckets=32, max_distance=128),
        _case("bias_one_token", "bias", 16, 24, 1, 2049, 64, ragged=True, buckets=32, max_distance=128,
              both_ways=False, causal=True, at_end=True),
        # Training it: a batch of prompts of odd length, and a decoder over a
        # long text.
        _case("bias_train_prompt", "bias_train", 8, 24, 226, 226, 64, layout="blhd", ragged=True, buckets=32,
              max_distance=128),
        _case("bias_train_long", "bias_train", 1, 12, 4095, 4095, 128, dtype="fp16", buckets=64, max_distance=500,
              both_ways=False, causal=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any kind, lengths over the whole range, every type, head
    size and layout; no more work than the long video's training step."""
    kind = rng.choice(["cross", "cross_train", "bias", "bias_train"])
    least = 8 if kind.endswith("train") else 1      # one key alone has no gradient but its value's
    D, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "fp16"])
    layout, ragged = rng.choice(["bhld", "blhd"]), rng.random() < 0.5
    B, H = rng.choice([1, 1, 2, 3, 4, 8]), rng.choice([2, 3, 6, 12, 24, 48])
    group = rng.choice([1, 1, 1, 2, 3, 6])
    kv = H // group if H % group == 0 else H
    more = dict(dtype=dtype, layout=layout, ragged=ragged, empty=ragged and rng.random() < 0.3,
                mask=rng.random() < 0.3)
    if kind.startswith("cross"):
        Lq, Lk = (_log(rng, 1, 110080), _log(rng, least, 512)) if rng.random() < 0.7 else \
            (_log(rng, 1, 256), _log(rng, 512, 110080))
    else:
        Lk = _log(rng, least, 8192 if kind == "bias" else 4096)
        more["both_ways"] = rng.random() < 0.6
        more["causal"] = not more["both_ways"]
        nb = rng.choice([8, 32, 64])
        more.update(buckets=nb, max_distance=rng.choice([64, 128, 500]), scale=rng.choice([0.0, 1.0]))
        Lq = Lk
        if kind == "bias" and not more["both_ways"] and rng.random() < 0.5:
            Lq, B = min(Lk, rng.choice([1, 1, 2, 5])), rng.choice([1, 4, 16, 32])
            more["at_end"] = True
    pairs, rows = 24 * 110080 * 256, 24 * 110080 * 128
    while B > 1 and (B * H * Lq * Lk > pairs or B * H * Lq * D > rows or B * kv * Lk * D > rows):
        B -= 1
    while H > 1 and (B * H * Lq * Lk > pairs or B * H * Lq * D > rows or B * kv * Lk * D > rows):
        H = kv = max(1, H // 2)
    return _case(None, kind, B, H, Lq, Lk, D, kv_heads=kv, **more)


def _lens(case):
    """Key lengths of the samples: the first has all keys, the others fewer;
    with ``empty`` the last has none.  None where every sample has all."""
    B, Lk = case["batch"], case["k_len"]
    if not case["ragged"]:
        return None
    lens = [max(1, Lk - (b * 5 * Lk) // (8 * B)) for b in range(B)]
    if case["at_end"]:
        lens = [max(n, case["q_len"]) for n in lens]
    if case["empty"] and B > 1 and not case["at_end"]:
        lens[-1] = 0
    return lens


# --- inputs ------------------------------------------------------------------

def prepare(case, seed):
    """Unit-variance queries and keys as normalised projections give them
    (scores of about unit variance), values with a mean of their own per
    channel, and for training the output's gradient."""
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + 77) % (1 << 62))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
    B, H, Hk, D = case["batch"], case["heads"], case["kv_heads"], case["head_dim"]

    def make(heads, length, std=1.0, mean=False):
        sh = (B, length, heads, D) if case["layout"] == "blhd" else (B, heads, length, D)
        t = torch.randn(sh, generator=g, device=DEV, dtype=torch.float32).mul_(std)
        t = t.transpose(1, 2) if case["layout"] == "blhd" else t
        if mean:
            t += 0.3 * torch.randn(1, heads, 1, D, generator=g, device=DEV)
        return t.to(dt)

    s = dict(case=case, lens=None, mask=None, table=None, dout=None)
    s["q"] = make(H, case["q_len"], D ** -0.5 if case["scale"] == 1.0 else 1.0)
    s["k"] = make(Hk, case["k_len"])
    s["v"] = make(Hk, case["k_len"], mean=True)
    if case["kind"].endswith("train"):
        s["dout"] = make(H, case["q_len"])
    lens = _lens(case)
    if lens is not None:
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if case["mask"]:
        s["mask"] = torch.rand(B, case["k_len"], generator=g, device=DEV) >= 0.125
    if case["buckets"]:
        s["table"] = (0.7 * torch.randn(case["buckets"], H, generator=g, device=DEV)).to(dt)
    return s


# --- the plain form ----------------------------------------------------------

def _bucket(rel, case):
    """The table row of each key position minus query position."""
    n_all, far = case["buckets"], case["max_distance"]
    nb = n_all // 2 if case["both_ways"] else n_all
    n = rel.abs() if case["both_ways"] else (-rel).clamp(min=0)
    e = nb // 2
    steps = torch.log(n.clamp(min=1).double() / e) / math.log(far / e) * (nb - e)
    b = torch.where(n < e, n, (e + torch.floor(steps + 1e-9).long()).clamp(max=nb - 1))
    return b + nb * (rel > 0) if case["both_ways"] else b


def _plain(s):
    c = s["case"]
    B, H, Hk, Lq, Lk, D = (c[x] for x in ("batch", "heads", "kv_heads", "q_len", "k_len", "head_dim"))
    G, dt = H // Hk, s["q"].dtype
    scale = c["scale"] or D ** -0.5
    q = s["q"].float().reshape(B, Hk, G * Lq, D)
    k, v = s["k"].float(), s["v"].float()
    j = torch.arange(Lk, device=DEV)
    seen = torch.ones(1, 1, 1, 1, Lk, dtype=torch.bool, device=DEV)
    if s["lens"] is not None:
        seen = seen & (j < s["lens"].view(B, 1, 1, 1, 1))
    if s["mask"] is not None:
        seen = seen & s["mask"].view(B, 1, 1, 1, Lk)
    x = (q @ k.transpose(-1, -2) * scale).view(B, Hk, G, Lq, Lk)
    if c["buckets"]:
        off = torch.zeros(1, device=DEV, dtype=torch.long)
        if c["at_end"]:
            off = (s["lens"].long() if s["lens"] is not None else off + Lk) - Lq
        rel = j - (torch.arange(Lq, device=DEV).view(1, Lq, 1) + off.view(-1, 1, 1))       # [1 or B, Lq, Lk]
        if c["causal"]:
            seen = seen & (rel <= 0)[:, None, None]
        x = x + s["table"].float()[_bucket(rel, c)].permute(0, 3, 1, 2).view(-1, Hk, G, Lq, Lk)
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    del x
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top).view(B, H, Lq)
    p = p / torch.where(total == 0, 1.0, total)
    flat = p.view(B, Hk, G * Lq, Lk)
    out = (flat @ v).view(B, H, Lq, D)
    if s["dout"] is None:
        return out.to(dt), lse
    do = s["dout"].float().reshape(B, Hk, G * Lq, D)
    dv = flat.transpose(-1, -2) @ do
    dx = do @ v.transpose(-1, -2)
    dx = flat * (dx - (flat * dx).sum(-1, keepdim=True))
    dq = (dx @ k * scale).view(B, H, Lq, D)
    dk = dx.transpose(-1, -2) @ q * scale
    grads = [out.to(dt), dq.to(dt), dk.to(dt), dv.to(dt)]
    if c["buckets"]:
        # Diagonals as columns: rows of Lk + Lq - 1 values laid end to end and
        # read as rows one longer shift back by one place each.
        d = dx.view(B, H, Lq, Lk).sum(0)
        d = torch.nn.functional.pad(d, (0, Lq - 1)).view(H, -1)
        d = torch.nn.functional.pad(d, (0, Lq)).view(H, Lq, Lk + Lq).sum(1)
        at = torch.arange(Lk + Lq, device=DEV)                     # column (j - i) mod (Lk + Lq)
        rel = torch.where(at < Lk, at, at - (Lk + Lq))
        dt_sum = torch.zeros(c["buckets"], H, device=DEV).index_add_(0, _bucket(rel, c), d.t().contiguous())
        grads.append(dt_sum.to(dt))
    return tuple(grads)


# --- one pass ----------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    import paper_2502_21079_amd as ad
    c = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    kw = dict(key_lens=s["lens"], key_mask=s["mask"], scale=c["scale"] or None)
    if c["buckets"]:
        kw.update(max_distance=c["max_distance"], bidirectional=c["both_ways"], causal=c["causal"],
                  q_offset="end" if c["at_end"] else 0)
        out, lse = ad.rel_bias_attn(q, k, v, s["table"], **kw)
        if s["dout"] is None:
            return out, lse
        return (out,) + ad.rel_bias_attn_bwd(s["dout"], q, k, v, s["table"], out, lse, **kw)
    out, lse = ad.cross_attn(q, k, v, **kw)
    if s["dout"] is None:
        return out, lse
    return (out,) + ad.cross_attn_bwd(s["dout"], q, k, v, out, lse, **kw)


def work(case):
    """Two products forward and four more backward (scores formed again are
    not counted), over the pairs that lengths and order leave visible; every
    input read and every output written once."""
    B, H, Hk, Lq, Lk, D = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "k_len", "head_dim"))
    train = case["kind"].endswith("train")
    lens = _lens(case) or [Lk] * B
    pairs = 0
    for n in lens:
        if not case["causal"]:
            pairs += Lq * n
            continue
        off = n - Lq if case["at_end"] else 0
        first = [min(n, max(0, off + 1)), min(n, max(0, off + Lq))]       # keys the first and the last query see
        full = Lq if first[0] == n else max(0, off + Lq - n)              # queries that see all n
        climb = Lq - full if first[0] < n else 0
        pairs += full * n + climb * (first[0] + min(first[1], n)) // 2
    rows, keys = B * H * Lq, Hk * sum(lens)
    moved = 2 * D * (2 * rows + 2 * keys) + 4 * rows
    if train:
        moved = 2 * D * (4 * rows + 2 * keys + 2 * B * Hk * Lk)           # q, dout; out, dq; k, v; dk, dv
    if case["buckets"]:
        moved += 2 * case["buckets"] * H * (2 if train else 1)
    return {"bytes": moved, "flops": (12 if train else 4) * H * pairs * D}


# --- 64 bits -----------------------------------------------------------------

def _exact_bucket(d, nb, far):
    """Bucket of distance d >= 0 among nb, by whole numbers: the step m of the
    logarithmic half is reached where (d / e)^(nb - e) >= (far / e)^m."""
    e = nb // 2
    if d < e:
        return d
    m = 0
    while m + 1 < nb - e and d ** (nb - e) * e ** (m + 1) >= far ** (m + 1) * e ** (nb - e):
        m += 1
    return e + m


def exact(case, seed):
    B, H, Hk, Lq, Lk, D = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "k_len", "head_dim"))
    s = prepare(case, seed)
    train, nb_all = s["dout"] is not None, case["buckets"]
    f8 = dict(dtype=torch.float64, device=DEV)
    scale = case["scale"] or 1.0 / math.sqrt(D)
    out, lse = torch.zeros(B, H, Lq, D, **f8), torch.full((B, H, Lq), -math.inf, **f8)
    if train:
        dq, dk, dv = torch.zeros(B, H, Lq, D, **f8), torch.zeros(B, Hk, Lk, D, **f8), torch.zeros(B, Hk, Lk, D, **f8)
        dtable = torch.zeros(max(1, nb_all), H, **f8)
    if nb_all:
        nb = nb_all // 2 if case["both_ways"] else nb_all
        far = max(Lq, Lk) + Lk
        near = [_exact_bucket(d, nb, case["max_distance"]) for d in range(min(far, case["max_distance"]) + 1)]
        by_distance = torch.tensor(near + [nb - 1] * (far + 1 - len(near)), device=DEV)
    lens = _lens(case) or [Lk] * B
    rows_at_once = max(1, (1 << 28) // max(1, Lk))
    for b in range(B):
        n = lens[b]
        keep = torch.arange(n, device=DEV)
        if s["mask"] is not None:
            keep = keep[s["mask"][b, :n]]
        if keep.numel() == 0:
            continue
        for h in range(H):
            k, v = s["k"][b, h // (H // Hk), keep].double(), s["v"][b, h // (H // Hk), keep].double()
            for r0 in range(0, Lq, rows_at_once):
                r = torch.arange(r0, min(Lq, r0 + rows_at_once), device=DEV)
                q = s["q"][b, h, r].double()
                x = torch.mm(q, k.t()) * scale
                if nb_all:
                    ahead = keep[None, :] - r[:, None] - (n - Lq if case["at_end"] else 0)
                    if case["both_ways"]:
                        at = by_distance[ahead.abs()] + nb * (ahead > 0)
                    else:
                        at = by_distance[(-ahead).clamp(min=0)]
                    x += s["table"][:, h].double()[at]
                    if case["causal"]:
                        x.masked_fill_(ahead > 0, -math.inf)
                lse[b, h, r] = z = torch.logsumexp(x, 1)
                p = torch.exp(x - torch.where(z.isinf(), torch.zeros_like(z), z)[:, None])
                out[b, h, r] = o = torch.mm(p, v)
                if not train:
                    continue
                do = s["dout"][b, h, r].double()
                dx = p * (torch.mm(do, v.t()) - (do * o).sum(1, keepdim=True))
                dq[b, h, r] = scale * torch.mm(dx, k)
                dk[b, h // (H // Hk)].index_add_(0, keep, scale * torch.mm(dx.t(), q))
                dv[b, h // (H // Hk)].index_add_(0, keep, torch.mm(p.t(), do))
                for u in range(nb_all):
                    dtable[u, h] += torch.where(at == u, dx, 0.0).sum()
    if not train:
        return out, lse
    return (out, dq, dk, dv) + ((dtable,) if nb_all else ())
