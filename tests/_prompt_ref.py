"""Plain 64-bit attention with key lengths, masks, shared key heads and a bias
by buckets, its gradients, and bounds on what a kernel may be off.

The bounds follow from the roundings that the kernels state: weights and dS
rounded to the inputs' type (relative u, and half a subnormal step), results
rounded once, the output used by the backward pass rounded, everything else in
fp32 (taken as 2e-5 of the sums of magnitudes: scores of up to about a hundred
log2 units and sums of up to 10^5 terms)."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SUB = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
FP32 = 2e-5


def starts_by_search(num_buckets, max_distance, bidirectional):
    """First distance of each bucket, from the bucket of every distance."""
    n = num_buckets // 2 if bidirectional else num_buckets
    e = n // 2

    def bucket(d):
        if d < e:
            return d
        m = 0
        while m + 1 < n - e and d ** (n - e) * e ** (m + 1) >= max_distance ** (m + 1) * e ** (n - e):
            m += 1
        return e + m
    of = [bucket(d) for d in range(max_distance + 1)]
    return [next(d for d in range(max_distance + 1) if of[d] >= m) for m in range(n)]


def bucket_index(rel, num_buckets, max_distance, bidirectional):
    """Table row of each key position minus query position."""
    starts = torch.tensor(starts_by_search(num_buckets, max_distance, bidirectional), device=rel.device)
    n = rel.abs() if bidirectional else (-rel).clamp(min=0)
    m = torch.searchsorted(starts, n.contiguous(), right=True) - 1
    return m + (len(starts) * (rel > 0) if bidirectional else 0)


def reference(q, k, v, *, dout=None, key_lens=None, key_mask=None, scale=None, table=None, max_distance=128,
              bidirectional=True, causal=False, q_offset=0, out_dtype=None):
    """dict of name -> (value, bound), all fp64; gradients where dout is given."""
    dt = out_dtype or q.dtype
    u, sub = U[dt], SUB[dt]
    B, H, Lq, D = q.shape
    Hk, Lk, dev = k.shape[1], k.shape[2], q.device
    G = H // Hk
    scale = scale or 1.0 / math.sqrt(D)
    q8 = q.double()
    seen = torch.ones(B, 1, Lq, Lk, dtype=torch.bool, device=dev)
    j = torch.arange(Lk, device=dev)
    lens = torch.full((B,), Lk, device=dev) if key_lens is None else key_lens.long().clamp(0, Lk)
    seen = seen & (j < lens.view(B, 1, 1, 1))
    if key_mask is not None:
        seen = seen & (key_mask != 0).view(B, 1, 1, Lk)
    any_key = seen.any(2).view(B, 1, Lk, 1)                     # keys that some row could see
    k8 = torch.where(any_key, k.double(), 0.0).repeat_interleave(G, 1)
    v8 = torch.where(any_key, v.double(), 0.0).repeat_interleave(G, 1)
    s = q8 @ k8.transpose(-1, -2) * scale
    if table is not None:
        off = (lens - Lq) if q_offset == "end" else torch.full((B,), int(q_offset), device=dev)
        rel = j.view(1, 1, Lk) - (torch.arange(Lq, device=dev).view(1, Lq, 1) + off.view(B, 1, 1))
        at = bucket_index(rel, table.shape[0], max_distance, bidirectional)
        s = s + table.double()[at].permute(0, 3, 1, 2)
        if causal:
            seen = seen & (rel <= 0).unsqueeze(1)
    s = torch.where(seen, s, -math.inf)
    lse = torch.logsumexp(s, -1) if Lk else torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device=dev)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse).unsqueeze(-1))
    out = p @ v8
    big = lambda t: float(t.abs().max()) if t.numel() else 0.0  # noqa: E731
    res = {"lse": (lse, FP32 * (1.0 + lse.abs())),
           "out": (out, u * out.abs() + (u + FP32) * (p @ v8.abs()) + Lk * sub * big(v8) + sub)}
    if dout is None:
        return res
    g8 = dout.double()
    dp = g8 @ v8.transpose(-1, -2)
    delta = (p * dp).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    # dS is off by the rounded output's share of delta, fp32 in P and dP, and its own rounding.
    d_err = (u + FP32) * (g8.abs() * (out.abs() + p @ v8.abs())).sum(-1, keepdim=True)
    e32 = p * (d_err + FP32 * (g8.abs() @ v8.abs().transpose(-1, -2)))
    es = e32 + u * ds.abs() + sub
    ep = (u + FP32) * p + sub

    def shared(t):
        return t.view(B, Hk, G, Lk, D).sum(2)
    dq, dk, dv = scale * (ds @ k8), scale * shared(ds.transpose(-1, -2) @ q8), shared(p.transpose(-1, -2) @ g8)
    es = torch.where(seen, es, 0.0)
    ep = torch.where(seen, ep, 0.0)
    res["dq"] = dq, u * dq.abs() + scale * (es @ k8.abs()) + sub
    res["dk"] = dk, u * dk.abs() + scale * shared(es.transpose(-1, -2) @ q8.abs()) + sub
    res["dv"] = dv, u * dv.abs() + shared(ep.transpose(-1, -2) @ g8.abs()) + sub
    if table is not None:
        rows = at.expand(B, Lq, Lk)
        dtab, e_tab = (torch.zeros(table.shape, dtype=torch.float64, device=dev) for _ in range(2))
        e32 = torch.where(seen, e32 + FP32 * ds.abs(), 0.0)
        for r in range(table.shape[0]):
            hit = (rows == r).unsqueeze(1)
            dtab[r] = torch.where(hit, ds, 0.0).sum((0, 2, 3))
            e_tab[r] = torch.where(hit, e32, 0.0).sum((0, 2, 3))
        ut = U.get(table.dtype, 2.0 ** -24)
        res["dtable"] = dtab, ut * dtab.abs() + e_tab + SUB.get(table.dtype, 0.0) + 1e-30
    return res


def check(got, ref, what):
    """Every entry within its bound; equal infinities."""
    val, bound = ref
    g = got.double()
    assert g.shape == val.shape, f"{what}: shape {tuple(g.shape)} for {tuple(val.shape)}"
    fin = torch.isfinite(val)
    assert torch.equal(torch.isfinite(g), fin), f"{what}: finite entries differ"
    assert torch.equal(g[~fin], val[~fin]), f"{what}: infinities differ"
    over = (g - val).abs()[fin] - bound[fin]
    assert not (over > 0).any(), (f"{what}: {int((over > 0).sum())} of {over.numel()} entries over their bound, worst by "
                                  f"{float(over.max()):.3e} (|ref| up to {float(val[fin].abs().max()):.3e})")
