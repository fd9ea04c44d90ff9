"""The serving operators together, as a program runs them: a batch whose sequences
share a prompt reads its questions in, then produces tokens one by one, with one
layer of full attention (kvcache_append_paged, fwd_prefix_paged) and one with a
sliding window (kvcache_append, fwd_window).  Every step is checked against the
definition in 64 bits on keys that a plain rotation in 64 bits has made; then the
token step is captured into graphs and replayed.

Tolerance: the caches hold keys rounded to bf16, and so does the reference (its
own rotation, rounded; a key may round the other way, by one place of 2^-8, in
some 10^-4 of the elements, which moves a score by less than 2^-8 |q| |k| scale <
0.02 in one of hundreds of keys); outputs as helpers.check_against."""
import pytest
import torch

import paper_2608_18656_amd as fa

from helpers import check_against

pytestmark = pytest.mark.gpu

B, HQ, HKV, D, P = 3, 8, 2, 64, 64
PREFIX, PAGES = 128, 6
WINDOW, SINKS = 40, 3
BF = torch.bfloat16


def rotate(x, pos, freq):
    """x [N, H, D] (bf16), pos [N]: the halves rotated, in 64 bits, rounded once."""
    t = pos.double()[:, None, None] * freq.double()
    a, b = x.double().chunk(2, -1)
    return torch.cat([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()], -1).to(x.dtype)


def attend(q, k, v, window=None):
    """q [N, HQ, D] the last N of k, v [n, HKV, D]: out [N, HQ, D] and lse [HQ, N] in 64 bits."""
    N, n = q.shape[0], k.shape[0]
    p, j = n - N + torch.arange(N)[:, None], torch.arange(n)[None]
    see = (j <= p) & ((j > p - window) | (j < SINKS)) if window else j <= p
    o, lse = torch.zeros(q.shape, dtype=torch.float64), torch.zeros((HQ, N), dtype=torch.float64)
    for h in range(HQ):
        g = h // (HQ // HKV)
        x = ((q[:, h].double() @ k[:, g].double().t()) * D ** -0.5).masked_fill(~see, -torch.inf)
        lse[h], o[:, h] = torch.logsumexp(x, 1), torch.softmax(x, 1) @ v[:, g].double()
    return o, lse


class Layers:
    """The caches of both layers on the GPU, and their contents on the CPU."""

    def __init__(self, seed=0):
        self.gen = torch.Generator().manual_seed(seed)
        self.freq = (1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float()
        self.dfreq = self.freq.cuda()
        own = PAGES - PREFIX // P
        perm = torch.randperm(PREFIX // P + B * own, generator=self.gen).int()
        shared = perm[:PREFIX // P].expand(B, -1)
        self.table = torch.cat([shared, perm[PREFIX // P:].view(B, own)], 1).contiguous().cuda()
        self.kp = torch.full((perm.numel(), P, HKV, D), float("nan"), dtype=BF, device="cuda")
        self.vp = self.kp.clone()
        self.kw = torch.full((B, 300, HKV, D), float("nan"), dtype=BF, device="cuda")
        self.vw = self.kw.clone()
        self.keys = [[torch.empty(0, HKV, D, dtype=BF) for _ in range(B)] for _ in range(2)]     # paged, window
        self.vals = [[torch.empty(0, HKV, D, dtype=BF) for _ in range(B)] for _ in range(2)]

    def fused(self, n):
        return torch.randn(B, n, (HQ + 2 * HKV) * D, generator=self.gen).to(BF)

    @staticmethod
    def parts(qkv):
        return [t.unflatten(2, (-1, D)) for t in qkv.split((HQ * D, HKV * D, HKV * D), 2)]

    def shared_prompt(self):
        """The prefix, read in once: sequence 0's table has its pages."""
        qkv = self.fused(PREFIX)[:1]
        q, k, v = self.parts(qkv.cuda())
        n = torch.tensor([PREFIX], dtype=torch.int32, device="cuda")
        fa.kvcache_append_paged(k, v, self.kp, self.vp, self.table[:1], n, q=q, inv_freq=self.dfreq)
        _, k, v = self.parts(qkv)
        for b in range(B):
            self.keys[0][b], self.vals[0][b] = rotate(k[0], torch.arange(PREFIX), self.freq), v[0]

    def remember(self, layer, qkv, new):
        """The reference's caches grow by each sequence's last new[b] tokens; its rotated queries."""
        q, k, v = self.parts(qkv)
        out = []
        for b, n in enumerate(new):
            have = self.keys[layer][b].shape[0]
            pos = torch.arange(have, have + n)
            if n:
                self.keys[layer][b] = torch.cat([self.keys[layer][b], rotate(k[b, -n:], pos, self.freq)])
                self.vals[layer][b] = torch.cat([self.vals[layer][b], v[b, -n:]])
            out.append(rotate(q[b, q.shape[1] - n:], pos, self.freq))
        return out

    def lengths(self, layer):
        return torch.tensor([k.shape[0] for k in self.keys[layer]], dtype=torch.int32, device="cuda")

    def step(self, qkv0, qkv1, n0, n1, ws=(None, None)):
        """Both layers' calls; n0, n1: lengths with the new tokens."""
        q, k, v = self.parts(qkv0)
        q = fa.kvcache_append_paged(k, v, self.kp, self.vp, self.table, n0, q=q, inv_freq=self.dfreq)
        full = fa.fwd_prefix_paged(q, self.kp, self.vp, self.table, n0, PREFIX, causal=True, workspace=ws[0])
        q, k, v = self.parts(qkv1)
        q = fa.kvcache_append(k, v, self.kw, self.vw, n1, q=q, inv_freq=self.dfreq)
        near = fa.fwd_window(q, self.kw, self.vw, WINDOW, sinks=SINKS, seqlens_k=n1, workspace=ws[1])
        return full, near

    def check(self, layer, got, queries, new, label):
        o, lse = got
        for b, n in enumerate(new):
            if n == 0:
                continue
            ref, rl = attend(queries[b], self.keys[layer][b], self.vals[layer][b], WINDOW if layer else None)
            check_against(o[b:b + 1, o.shape[1] - n:], lse[b:b + 1, :, o.shape[1] - n:], ref[None].numpy(), rl[None].numpy(), BF,
                          False, f"{label} b={b}")


@pytest.mark.parametrize("chunk", [20, 40])
def test_prompt_and_tokens(chunk):
    s = Layers(chunk)
    s.shared_prompt()
    # the questions, of different lengths: padded in front
    new = [chunk, chunk - 7, 5]
    qkv0, qkv1 = s.fused(chunk), s.fused(chunk)
    qs0, qs1 = s.remember(0, qkv0, new), s.remember(1, qkv1, new)
    # padding tokens of the paged layer would lie in the prefix: the program gives them no place
    n0 = s.lengths(0)
    got = []
    for b in range(B):
        one = qkv0[b:b + 1, chunk - new[b]:].cuda()
        q, k, v = s.parts(one)
        q = fa.kvcache_append_paged(k, v, s.kp, s.vp, s.table[b:b + 1], n0[b:b + 1], q=q, inv_freq=s.dfreq)
        got.append(fa.fwd_prefix_paged(q, s.kp, s.vp, s.table[b:b + 1], n0[b:b + 1], PREFIX, causal=True))
    for b in range(B):
        ref, rl = attend(qs0[b], s.keys[0][b], s.vals[0][b])
        check_against(*got[b], ref[None].numpy(), rl[None].numpy(), BF, False, f"question {b}")
    q, k, v = s.parts(qkv1.cuda())
    n1 = s.lengths(1)
    q = fa.kvcache_append(k, v, s.kw, s.vw, n1, q=q, inv_freq=s.dfreq)   # rows below 0 are padding
    s.check(1, fa.fwd_window(q, s.kw, s.vw, WINDOW, sinks=SINKS, seqlens_k=n1), qs1, new, "window question")
    # tokens: past the edges of pages and of the window
    for t in range(60):
        qkv0, qkv1 = s.fused(1), s.fused(1)
        qs0, qs1 = s.remember(0, qkv0, [1] * B), s.remember(1, qkv1, [1] * B)
        full, near = s.step(qkv0.cuda(), qkv1.cuda(), s.lengths(0), s.lengths(1))
        s.check(0, full, qs0, [1] * B, f"token {t}")
        s.check(1, near, qs1, [1] * B, f"window token {t}")


def _prompted(seed):
    s = Layers(seed)
    s.shared_prompt()
    qkv = s.fused(50)
    for layer in range(2):
        s.remember(layer, qkv, [50] * B)
    s.step(qkv.cuda(), qkv.cuda(), s.lengths(0), s.lengths(1))
    return s


def _workspaces():
    need = (fa.prefix_workspace_bytes(B, HQ, HKV, 1, PREFIX, PAGES * P - PREFIX, D, "bf16"),
            fa.window_workspace_bytes(B, HQ, HKV, 1, 300, D, WINDOW, "bf16", sinks=SINKS))
    return tuple(torch.empty(n, dtype=torch.uint8, device="cuda") for n in need)


def _captured(s, ws):
    """The token step as a graph: (graph, its inputs, its outputs).  s keeps ws, which the graph uses."""
    s.workspaces = ws
    qkv = [torch.zeros(B, 1, (HQ + 2 * HKV) * D, dtype=BF, device="cuda") for _ in range(2)]
    n = [s.lengths(0), s.lengths(1)]
    for x in n:
        x += 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step(*qkv, *n, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = s.step(*qkv, *n, ws)
    torch.cuda.synchronize()
    return graph, qkv, n, out


def test_graph_replays_equal_eager():
    """Replays, with eager work between them, give what the eager calls give on caches of the same contents."""
    s, e = _prompted(1), _prompted(1)
    graph, qkv, n, out = _captured(s, _workspaces())
    for rep in range(5):
        new = [e.fused(1).cuda(), e.fused(1).cuda()]
        at = [torch.tensor([x.shape[0] + 1 + rep for x in e.keys[layer]], dtype=torch.int32, device="cuda") for layer in range(2)]
        eager = [t.clone() for pair in e.step(*new, *at) for t in pair]
        for dst, src in zip((*qkv, *n), (*new, *at)):
            dst.copy_(src)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((t for pair in out for t in pair), eager):
            assert torch.equal(a, b), f"replay {rep}"
        assert torch.equal(s.kp.view(torch.int16), e.kp.view(torch.int16))
        assert torch.equal(s.vw.view(torch.int16), e.vw.view(torch.int16))


def test_two_graphs_at_once():
    """Two captured steps with workspaces of their own, replayed on two streams at the same time."""
    runs = []
    for seed in (3, 4):
        s = _prompted(seed)
        runs.append((s, *_captured(s, _workspaces())))
    new = [[s.fused(1).cuda() for _ in range(2)] for s, *_ in runs]
    for (s, graph, qkv, n, out), x in zip(runs, new):
        for dst, src in zip(qkv, x):
            dst.copy_(src)
    alone = []
    for s, graph, qkv, n, out in runs:
        graph.replay()
        torch.cuda.synchronize()
        alone.append([t.clone() for pair in out for t in pair])
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(4):
        for (s, graph, qkv, n, out), st in zip(runs, streams):
            with torch.cuda.stream(st):
                for _ in range(5):
                    graph.replay()
        torch.cuda.synchronize()
        for (s, graph, qkv, n, out), ref in zip(runs, alone):
            for a, b in zip((t for pair in out for t in pair), ref):
                assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls on two streams, each with the library's workspace of its stream, equal the same calls one after the other."""
    q = [torch.randn(8, 1, 32, 128, device="cuda").to(BF) for _ in range(2)]
    k = [torch.randn(8, 3000, 8, 128, device="cuda").to(BF) for _ in range(2)]
    kp = [torch.randn(2000, 8, 128, device="cuda").to(BF) for _ in range(2)]
    calls = [lambda i=i: (fa.fwd_prefix(q[i], kp[i], kp[i], k[i], k[i]), fa.fwd_window(q[i], k[i], k[i], 2500, sinks=9)) for i in range(2)]
    ref = [[[t.clone() for t in pair] for pair in c()] for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for c, st in zip(calls, streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append([c() for _ in range(6)])
        torch.cuda.synchronize()
        for runs, want in zip(got, ref):
            for run in runs:
                for pair, w in zip(run, want):
                    assert all(torch.equal(a, b) for a, b in zip(pair, w))


def test_set_workspace_serves_and_refuses():
    q, kp, k = (torch.randn(s, device="cuda").to(BF) for s in ((4, 1, 32, 128), (3000, 8, 128), (4, 900, 8, 128)))
    ref = fa.fwd_prefix(q, kp, kp, k, k)[0].clone()
    need = fa.prefix_workspace_bytes(4, 32, 8, 1, 3000, 900, 128, "bf16")
    try:
        fa.set_workspace(torch.empty(need, dtype=torch.uint8, device="cuda"))
        assert torch.equal(fa.fwd_prefix(q, kp, kp, k, k)[0], ref)
        fa.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
        with pytest.raises(fa.FaError) as e:
            fa.fwd_prefix(q, kp, kp, k, k)
        assert e.value.status == 10
        fa.fwd_prefix(q, kp[:20], kp[:20], k[:, :20].contiguous(), k[:, :20].contiguous(), causal=True)   # one pass needs none
    finally:
        fa.set_workspace(None)
    torch.cuda.synchronize()


def test_bitwise_determinism():
    q, kp, k = (torch.randn(s, device="cuda").to(BF) for s in ((16, 1, 32, 128), (5000, 8, 128), (16, 700, 8, 128)))
    a = fa.fwd_prefix(q, kp, kp, k, k)
    for _ in range(5):
        b = fa.fwd_prefix(q, kp, kp, k, k)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_outgrown_workspace_is_the_streams_own_from_then_on():
    """A stream's library-owned workspace, outgrown by larger calls on several streams, is the larger one
    from then on: the same calls are captured (where nothing may be allocated) and replay the eager results."""
    gen = torch.Generator("cuda").manual_seed(11)
    kp, vp = (torch.randn(1000, 4, 128, generator=gen, device="cuda", dtype=BF) for _ in range(2))
    calls = []
    for n in (1, 40):
        q, k, v = (torch.randn(n, m, h, 128, generator=gen, device="cuda", dtype=BF) for m, h in ((1, 16), (90, 4), (90, 4)))
        calls.append((q, kp, vp, k, v))
    assert fa.prefix_workspace_bytes(1, 16, 4, 1, 1000, 90, 128, "bf16") < 1 << 20
    assert fa.prefix_workspace_bytes(40, 16, 4, 1, 1000, 90, 128, "bf16") > 1 << 20
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    eager = []
    for small_or_large in calls:
        for st in streams:
            with torch.cuda.stream(st):
                eager.append(fa.fwd_prefix(*small_or_large))
    torch.cuda.synchronize()
    for st, (o, lse) in zip(streams, eager[3:]):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            og, lg = fa.fwd_prefix(*calls[1])
        for _ in range(3):
            og.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(og, o) and torch.equal(lg, lse)
