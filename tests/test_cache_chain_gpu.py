"""Rotary positions, writing and attention together, as a decoder runs them: prompts
of different lengths, then single tokens, also captured in a graph, against the
definitions in 64 bits."""
import pytest
import torch

import paper_2502_21079_amd as ad
from _cache_ref import SUB, U, Sequences, attn_reference, rotary_reference, within

pytestmark = pytest.mark.gpu

DEV = "cuda"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Layer:
    """One attention layer with its cache: projections are what :meth:`tokens` draws."""

    def __init__(self, B, H, Hk, D, page, most, dt, layout):
        self.B, self.H, self.Hk, self.D, self.dt = B, H, Hk, D, dt
        cap = -(-most // page)
        g = torch.Generator().manual_seed(B + D)
        self.cache = ad.kv_cache(B * cap + 1, Hk, page, D)
        self.table = torch.randperm(B * cap + 1, generator=g)[:B * cap].view(B, cap).to(torch.int32).to(DEV)
        self.before, self.after = i32([0] * B), i32([0] * B)
        self.rope = dict(freqs=ad.rotary_frequencies(D // 2, scaling="linear", factor=2.0), layout=layout)

    def tokens(self, T, seed):
        g = torch.Generator().manual_seed(seed)
        qkv = torch.randn(self.B, T, self.H + 2 * self.Hk, self.D, generator=g).to(self.dt).to(DEV).transpose(1, 2)
        return qkv[:, :self.H], qkv[:, self.H:self.H + self.Hk], qkv[:, self.H + self.Hk:]

    def step(self, q, k, v, new=None, **out):
        """New tokens of each sequence attend to what is there and to themselves."""
        q, k = ad.rotary(q, k, offset=self.before, **self.rope)
        ad.cache_write(k, v, self.cache, self.table, self.before, new_lens=new)
        self.after.copy_(self.before + (q.shape[2] if new is None else new))
        o, lse = ad.cache_attn(q, self.cache, self.table, self.after, q_lens=new, **out)
        self.before.copy_(self.after)
        return o, lse


@pytest.mark.parametrize("dt,D,page,layout", [(torch.bfloat16, 128, 64, "half"), (torch.float16, 64, 16, "interleaved"),
                                              (torch.bfloat16, 64, 128, "interleaved")])
def test_prompts_then_tokens(dt, D, page, layout):
    B, H, Hk = 3, 4, 2
    layer, seqs, lens = Layer(B, H, Hk, D, page, 400, dt, layout), Sequences(B, Hk, page, D), [0] * B
    steps = [(150, [150, 3, 77]), (40, [0, 40, 11])] + [(1, None)] * 5
    for i, (T, new) in enumerate(steps):
        q, k, v = layer.tokens(T, 10 * i)
        out, lse = layer.step(q, k, v, None if new is None else i32(new))
        # The cache holds what the definition makes of the turned keys that the kernel gave.
        qr, kr = ad.rotary(q, k, offset=i32(lens), **layer.rope)
        for x, y, n in ((q, qr, "q"), (k, kr, "k")):
            ref, bound = rotary_reference(x, layer.rope["freqs"], layout=layout, offset=lens)
            within(y, (ref, bound + U[dt] * ref.abs() + SUB[dt]), n)
        for b in range(B):
            n = T if new is None else new[b]
            seqs.write(b, kr[b, :, :n], v[b, :, :n])
            lens[b] += n
        assert layer.before.tolist() == lens
        ref = attn_reference(qr, seqs.x[0], seqs.x[1], lens, q_lens=new)
        within(out, ref["out"], f"out of step {i}")
        within(lse, ref["lse"], f"lse of step {i}")
    k, v = ad.cache_read(layer.cache, layer.table, i32(lens), max(lens))
    for b in range(B):
        assert torch.equal(k[b, :, :lens[b]].cpu().double(), seqs.x[0][b])
        assert torch.equal(v[b, :, :lens[b]].cpu().double(), seqs.x[1][b])


def test_a_captured_step_follows_the_lengths():
    """One token of each sequence, captured once: replays walk on through the pages and
    equal the same steps run eagerly, bit for bit, with eager work between them."""
    B, H, Hk, D, page = 2, 6, 2, 128, 32
    eager, graph = (Layer(B, H, Hk, D, page, 3000, torch.bfloat16, "half") for _ in range(2))
    for layer in (eager, graph):
        layer.step(*layer.tokens(90, 1), i32([90, 61]))
    q, k, v = graph.tokens(1, 2)
    out, lse = torch.empty_like(q), torch.empty(B, H, 1, device=DEV)
    ws = torch.empty(ad.cache_attn_workspace(q.shape, graph.cache, graph.table.shape[1]), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    saved = graph.before.clone()
    with torch.cuda.stream(side):
        graph.step(q, k, v, out=out, lse=lse, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph.before.copy_(saved)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graph.step(q, k, v, out=out, lse=lse, workspace=ws)
    graph.before.copy_(saved)
    for step in range(40):
        new = eager.tokens(1, 100 + step)
        for a, b in zip((q, k, v), new):
            a.copy_(b)
        want, wl = eager.step(*new)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl), step
        assert graph.before.tolist() == eager.before.tolist()
    for a, b in ((graph.cache.k, eager.cache.k), (graph.cache.v, eager.cache.v)):
        ids = graph.table[:, :90 // page].flatten().long()
        assert torch.equal(a.view(torch.uint8)[ids], b.view(torch.uint8)[ids])


def test_what_is_read_back_serves_the_other_attentions():
    """The cache's keys and values through cross_attn: the same numbers within both bounds."""
    B, H, Hk, D = 2, 4, 2, 64
    layer = Layer(B, H, Hk, D, 32, 600, torch.bfloat16, "half")
    layer.step(*layer.tokens(500, 3), i32([500, 300]))
    q, _, _ = layer.tokens(7, 4)
    lens = i32([500, 300])
    out, lse = ad.cache_attn(q, layer.cache, layer.table, lens, causal=False)
    k, v = ad.cache_read(layer.cache, layer.table, lens, 500)
    out2, lse2 = ad.cross_attn(q, k, v, key_lens=lens)
    ks, vs = [k[b, :, :n] for b, n in enumerate((500, 300))], [v[b, :, :n] for b, n in enumerate((500, 300))]
    ref = attn_reference(q, ks, vs, [500, 300], causal=False)
    for o, z in ((out, lse), (out2, lse2)):
        within(o, ref["out"], "out")
        within(z, ref["lse"], "lse")
