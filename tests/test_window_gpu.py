"""fwd_window and fwd_window_paged against the definition in 64 bits: key j is
visible to the query at position p iff j <= p and (j > p - window or j < sinks).

Keys that no query of a sequence sees hold NaN and infinities here, and table
entries of pages without a visible key name no page or one full of NaN.  The
tolerance is that of the attention forward (helpers.check_against)."""
import random

import pytest
import torch

import paper_2608_18656_amd as fa
from paper_2608_18656_amd.inputs import DTYPES, make_qkv

from helpers import check_against, default_scale

pytestmark = pytest.mark.gpu


def visible(Nq, n, Nk, window, sinks):
    """[Nq, Nk]: what the last Nq positions of a sequence of n keys see."""
    p = n - Nq + torch.arange(Nq)[:, None]
    j = torch.arange(Nk)[None]
    return (j <= p) & ((j > p - window) | (j < sinks))


def reference(q, k, v, lens, window, sinks, scale):
    """float64 out [B, Nq, Hq, D] and lse [B, Hq, Nq]; rows without a key give 0 and -inf."""
    B, Nq, Hq, D = q.shape
    Nk, Hkv = k.shape[1:3]
    o, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full((B, Hq, Nq), -torch.inf, dtype=torch.float64)
    for b in range(B):
        see = visible(Nq, lens[b], Nk, window, sinks)
        rows = see.any(1)
        if not rows.any():
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            x = (q[b, :, h].double() @ k[b, :, g].double().t()) * scale
            x = x.masked_fill(~see, -torch.inf)[rows]
            lse[b, h, rows] = torch.logsumexp(x, 1)
            o[b, rows, h] = torch.softmax(x, 1) @ v[b, :, g].double()
    return o.numpy(), lse.numpy()


def poison(k, v, lens, Nq, window, sinks, seed):
    """k and v with NaN and infinities where no query sees them, and what is seen [B, Nk]."""
    k, v = k.clone(), v.clone()
    seen = torch.stack([visible(Nq, n, k.shape[1], window, sinks).any(0) for n in lens])
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=k.dtype)
    gen = torch.Generator().manual_seed(seed)
    for t in (k, v):
        t[~seen] = bad[torch.randint(0, 3, t[~seen].shape, generator=gen)]
    return k, v, seen


def paginate(k, v, seen, P, seed):
    """Pools and table; entries of blocks without a seen key lie outside the pool or name a page of NaN."""
    B, Nk, Hkv, D = k.shape
    n = -(-Nk // P)
    gen = torch.Generator().manual_seed(seed)
    perm = torch.randperm(B * n + 1, generator=gen).int()
    table = perm[:B * n].view(B, n).clone()
    pools = []
    for t in (k, v):
        pool = torch.full((B * n + 1, P, Hkv, D), float("nan"), dtype=t.dtype)
        rows = torch.full((B, n * P, Hkv, D), float("nan"), dtype=t.dtype)
        rows[:, :Nk] = t
        pool[table.long().view(-1)] = rows.view(B * n, P, Hkv, D)
        pools.append(pool)
    full = torch.zeros((B, n * P), dtype=torch.bool)
    full[:, :Nk] = seen
    used = full.view(B, n, P).any(2)
    other = torch.where(torch.arange(n) % 2 == 0, perm[-1], torch.tensor(1 << 30, dtype=torch.int32)).expand(B, n)
    return pools[0], pools[1], torch.where(used, table, other).int().contiguous()


def check_case(B, Hq, Hkv, Nq, Nk, D, dt, window, sinks, lens, page, seed=3, scale=None):
    q, k, v = make_qkv(B, Hq, Hkv, Nq, Nk, D, dt, seed=seed)
    scale = default_scale(D) if scale is None else scale
    n = lens if lens is not None else [Nk] * B
    ref = reference(q, k, v, n, window, sinks, scale)
    kp, vp, seen = poison(k, v, n, Nq, window, sinks, seed)
    sl = torch.tensor(n, dtype=torch.int32, device="cuda") if lens is not None or page else None
    if page:
        kp, vp, table = paginate(kp, vp, seen, page, seed)
        call = lambda odt, **kw: fa.fwd_window_paged(q.cuda(), kp.cuda(), vp.cuda(), table.cuda(), sl, window,   # noqa: E731
                                                     sinks=sinks, scale=scale, out_dtype=odt, **kw)
    else:
        call = lambda odt, **kw: fa.fwd_window(q.cuda(), kp.cuda(), vp.cuda(), window, sinks=sinks, seqlens_k=sl,   # noqa: E731
                                               scale=scale, out_dtype=odt, **kw)
    for odt in {torch.float32, DTYPES[dt]}:
        o, lse = call(odt)
        torch.cuda.synchronize()
        none = torch.isneginf(torch.from_numpy(ref[1]))
        assert torch.equal(torch.isneginf(lse.cpu()), none)
        assert bool((o.cpu().transpose(1, 2)[none] == 0).all())
        ok = torch.where(none, 0.0, lse.cpu().double()), torch.where(none, 0.0, torch.from_numpy(ref[1]))
        check_against(o, ok[0], ref[0], ok[1].numpy(), DTYPES[dt], odt == torch.float32,
                      f"window {B, Hq, Hkv, Nq, Nk, D, dt, window, sinks, lens, page, odt}")


EDGES = [
    # one token: lengths of 0 and 1, shorter and longer than the window, one split and many
    (5, 32, 8, 1, 700, 128, "bf16", 100, 4, [700, 0, 1, 104, 90], 0),
    (5, 32, 8, 1, 700, 64, "f16", 100, 4, [700, 0, 1, 104, 90], 64),
    (1, 16, 1, 1, 9000, 64, "f16", 4096, 4, [8999], 0),
    (2, 4, 4, 1, 5000, 128, "f16", 1, 0, [5000, 3], 64),
    (2, 40, 2, 1, 5000, 128, "bf16", 33, 129, [4999, 130], 128),
    (3, 8, 2, 1, 300, 64, "bf16", 10000, 0, [300, 299, 5], 0),            # a window past every cache
    (1, 8, 2, 1, 300, 64, "bf16", 7, 10000, None, 0),                     # more sinks than keys
    (70, 8, 8, 1, 2000, 64, "bf16", 640, 0, [2000 - 13 * i for i in range(70)], 64),
    # prompts: windows and sinks at the edges of tiles
    (1, 8, 2, 300, 300, 64, "bf16", 1, 0, None, 0),
    (1, 8, 2, 300, 300, 128, "f16", 32, 1, None, 0),
    (2, 4, 4, 257, 257, 64, "f16", 33, 31, None, 0),
    (1, 4, 4, 390, 390, 128, "bf16", 65, 33, None, 0),
    (1, 6, 3, 450, 450, 64, "bf16", 64, 64, None, 0),
    (1, 3, 1, 450, 450, 128, "f16", 63, 100, None, 0),
    (1, 2, 2, 700, 700, 64, "f16", 700, 5, None, 0),
    (1, 16, 1, 1100, 1100, 64, "f16", 200, 300, None, 0),
    # chunks against caches of their own lengths, shorter than the chunk among them
    (4, 8, 2, 70, 900, 64, "bf16", 128, 4, [900, 33, 0, 500], 0),
    (4, 8, 2, 70, 900, 128, "bf16", 128, 4, [900, 33, 0, 500], 64),
    (3, 32, 8, 5, 640, 128, "f16", 90, 70, [640, 4, 200], 128),
    (2, 8, 8, 40, 10000, 64, "f16", 1000, 200, [10000, 9000], 64),        # tables of more than 64 pages, crossed in the window
    (1, 8, 8, 33, 9000, 128, "bf16", 4500, 4300, [8990], 64),             # and in the sinks
    (2, 4, 1, 2, 66, 64, "f16", 2, 1, [66, 1], 0),
    # few row blocks and long windows: tiles split over workgroups; splits that begin in the sinks, in the window, with nothing
    (2, 8, 2, 8, 9000, 128, "bf16", 4096, 4, [9000, 5000], 0),
    (2, 8, 2, 8, 9000, 64, "f16", 4096, 700, [9000, 5], 64),
    (1, 4, 4, 40, 9000, 128, "f16", 3000, 4000, [8200], 64),
    (1, 16, 2, 33, 6000, 64, "bf16", 2500, 1, None, 0),
    (3, 4, 1, 5, 5000, 128, "bf16", 5000, 0, [5000, 3, 0], 128),
    (1, 3, 3, 200, 6000, 64, "bf16", 5900, 70, [5999], 0),
    # fp32 weights: fp32 inputs and other head sizes
    (2, 4, 2, 1, 333, 64, "f32", 50, 3, [333, 20], 0),
    (2, 4, 2, 100, 333, 40, "f32", 50, 3, [333, 60], 0),
    (1, 16, 2, 250, 250, 128, "f32", 64, 17, None, 0),
    (1, 4, 4, 200, 200, 256, "f32", 31, 0, None, 0),
    (2, 8, 2, 77, 400, 96, "bf16", 100, 5, [400, 50], 0),
    (3, 8, 2, 1, 400, 80, "f16", 100, 5, [400, 50, 0], 0),
    (1, 8, 8, 300, 300, 160, "f16", 3, 40, None, 0),
    (1, 32, 8, 600, 600, 256, "bf16", 129, 1, None, 0),
    (1, 8, 8, 400, 400, 8, "bf16", 70, 70, None, 0),
]


@pytest.mark.parametrize("case", EDGES, ids=lambda c: "-".join(str(x) for x in c[:9]) + f"-{c[10]}")
def test_edges(case):
    check_case(*case)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
@pytest.mark.parametrize("Nq,D,dt", [(1, 64, "bf16"), (80, 128, "f16"), (80, 64, "bf16"), (30, 72, "f32")])
def test_scales(scale, Nq, D, dt):
    check_case(2, 8, 2, Nq, 500, D, dt, 90, 6, [500, 300], 0, scale=scale)


def _random_case(seed):
    r = random.Random(seed)
    dt = r.choice(("bf16", "f16", "bf16", "f16", "f32"))
    page = r.choice((0, 0, 64, 128)) if dt != "f32" else 0
    D = r.choice((64, 128)) if page or r.random() < 0.7 else 8 * r.randint(1, 32)
    Hkv = r.choice((1, 2, 3, 8))
    Hq, B = Hkv * r.choice((1, 2, 4, 5, 8, 17)), r.randint(1, 4)
    Nk = r.choice((r.randint(1, 100), r.randint(100, 1500)))
    Nq = r.choice((1, r.randint(1, min(Nk, 200))))
    lens = None if r.random() < 0.3 and not page else [r.choice((r.randint(0, Nk), r.randint(Nk // 2, Nk))) for _ in range(B)]
    window = r.choice((1, r.randint(1, 100), r.randint(1, Nk), 32 * r.randint(1, 8), 2 ** 31 - 1))
    return B, Hq, Hkv, Nq, Nk, D, dt, window, r.choice((0, 0, r.randint(1, 8), r.randint(1, 200), 32 * r.randint(0, 4))), lens, page, seed


@pytest.mark.parametrize("seed", range(40))
def test_random(seed):
    check_case(*_random_case(seed))


def test_a_window_of_one_is_the_row_itself():
    q, k, v = (t.cuda() for t in make_qkv(2, 8, 2, 200, 200, 64, "bf16", seed=1))
    o, _ = fa.fwd_window(q, k, v, 1)
    assert torch.equal(o.view(2, 200, 2, 4, 64), v[:, :, :, None].expand(2, 200, 2, 4, 64))
    o, _ = fa.fwd_window(q[:, :1].contiguous(), k, v, 1)
    assert torch.equal(o.view(2, 2, 4, 64), v[:, -1, :, None].expand(2, 2, 4, 64))


def test_a_window_of_all_keys_is_causal_attention():
    for Nq, D in ((1, 64), (1, 128), (150, 64), (150, 128)):
        q, k, v = (t.cuda() for t in make_qkv(2, 8, 2, Nq, 777, D, "f16", seed=2))
        n = torch.tensor([777, 400], dtype=torch.int32, device="cuda")
        a, la = fa.fwd_kvcache(q, k, v, n, causal=True, out_dtype=torch.float32)
        b, lb = fa.fwd_window(q, k, v, 777, seqlens_k=n, out_dtype=torch.float32)
        # the same weights in fp16 and sums in fp32, split elsewhere at most: twice the weights' rounding, 2^-11 of |v| <= 6
        assert float((a - b).abs().max()) <= 6 * 2.0 ** -11 and float((la - lb).abs().max()) <= 2.0 ** -11


def test_long_cache_rows_past_31_bits():
    """Windows at the end of caches of more than 2^31 elements and 4 GiB."""
    Nk, Hkv, D = 300_000, 64, 128
    k = torch.zeros((1, Nk, Hkv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    k[:, -200:], v[:, -200:] = torch.randn_like(k[:, -200:]), torch.randn_like(v[:, -200:])
    for Nq in (1, 50):
        q = torch.randn((1, Nq, Hkv, D), device="cuda").to(torch.bfloat16)
        a, la = fa.fwd_window(q, k, v, 100, out_dtype=torch.float32)
        b, lb = fa.fwd_window(q, k[:, -200:].contiguous(), v[:, -200:].contiguous(), 100, out_dtype=torch.float32)
        assert float((a - b).abs().max()) <= 6 * 2.0 ** -11 and float((la - lb).abs().max()) <= 2.0 ** -11


def test_parts_workspace():
    """Row blocks split over workgroups: with a workspace of the call's own, too small a one, and the library's."""
    q, k, v = (t.cuda() for t in make_qkv(1, 32, 8, 9, 8000, 128, "bf16", seed=8))
    need = fa.window_workspace_bytes(1, 32, 8, 9, 8000, 128, 4000, "bf16", sinks=4)
    assert need > 0
    ref, lse = fa.fwd_window(q, k, v, 4000, sinks=4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    mine, mlse = fa.fwd_window(q, k, v, 4000, sinks=4, workspace=ws)
    assert torch.equal(ref, mine) and torch.equal(lse, mlse)
    with pytest.raises(fa.FaError) as e:
        fa.fwd_window(q, k, v, 4000, sinks=4, workspace=ws[:1024])
    assert e.value.status == 10
    for Nk in (9, 40, 500, 3000, 4100):
        fa.fwd_window(q, k[:, :Nk].contiguous(), v[:, :Nk].contiguous(), 4000, sinks=4, workspace=ws)
    torch.cuda.synchronize()


def test_workspaces():
    q, k, v = (t.cuda() for t in make_qkv(4, 32, 8, 1, 5000, 128, "bf16", seed=4))
    need = fa.window_workspace_bytes(4, 32, 8, 1, 5000, 128, 2048, "bf16", sinks=4)
    assert 0 < need <= fa.workspace_bytes(4, 32, 8, 1, 5000, 128, "bf16")
    ref, lse = fa.fwd_window(q, k, v, 2048, sinks=4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    mine, mlse = fa.fwd_window(q, k, v, 2048, sinks=4, workspace=ws)
    assert torch.equal(ref, mine) and torch.equal(lse, mlse)
    with pytest.raises(fa.FaError) as e:
        fa.fwd_window(q, k, v, 2048, sinks=4, workspace=ws[:need - 16])
    assert e.value.status == 10
    # serves every shorter cache
    for Nk in (1, 31, 500, 2047, 2053, 4000):
        fa.fwd_window(q, k[:, :Nk].contiguous(), v[:, :Nk].contiguous(), 2048, sinks=4, workspace=ws)
    torch.cuda.synchronize()


@pytest.mark.parametrize("D,H,Nq", [(128, 270601, 1), (128, 270601, 4), (64, 270601, 3)])
def test_key_rows_past_32_bit_offsets(D, H, Nq):
    """Tiles of more than 2 GiB, contiguous and in pages of which the middle one is not seen."""
    gen = torch.Generator("cuda").manual_seed(6)
    Nk, W, S = 160, 20, 2
    k, v = (torch.randn(1, 192, H, D, generator=gen, device="cuda", dtype=torch.float16) for _ in range(2))
    q = torch.randn(1, Nq, H, D, generator=gen, device="cuda", dtype=torch.float16)
    n = torch.tensor([Nk], dtype=torch.int32, device="cuda")
    o, lse = fa.fwd_window(q, k, v, W, sinks=S, seqlens_k=n, out_dtype=torch.float32)
    table = torch.tensor([[0, 1 << 20, 2]], dtype=torch.int32, device="cuda")
    op, lp = fa.fwd_window_paged(q, k.view(3, 64, H, D), v.view(3, 64, H, D), table, n, W, sinks=S, out_dtype=torch.float32)
    assert torch.equal(o, op) and torch.equal(lse, lp)
    for h0 in range(0, H, 16384):
        h = slice(h0, h0 + 16384)
        for i in range(Nq):
            p = Nk - Nq + i
            see = list(range(S)) + list(range(p - W + 1, p + 1))
            w = torch.softmax((q[0, i, h].double() * k[0, see, h].double()).sum(-1) * default_scale(D), 0)
            ref = (w[:, :, None] * v[0, see, h].double()).sum(0)
            assert (o[0, i, h].double() - ref).abs().max().item() <= 2e-3, (h0, i)


@pytest.mark.parametrize("window,sinks", [(1, 1), (5, 3), (17, 1), (40, 30), (33, 33), (20, 64), (70, 65), (31, 95), (64, 0)])
@pytest.mark.parametrize("D,dt,Hq,Hkv", [(64, "f16", 4, 1), (64, "bf16", 6, 2), (128, "f16", 3, 3), (128, "bf16", 4, 1)])
def test_the_last_sink_and_the_window_in_one_tile(D, dt, Hq, Hkv, window, sinks):
    """Row blocks whose window begins in the tile of the last sink, next to it, and further on."""
    check_case(1, Hq, Hkv, 230, 230, D, dt, window, sinks, None, 0)
    check_case(2, Hq, Hkv, 100, 230, D, dt, window, sinks, [230, 131], 64)


@pytest.mark.parametrize("D,Nk,window,page", [(64, 1000, 600, 0), (128, 900, 900, 0), (128, 1000, 500, 64)])
def test_sequences_taken_by_length(D, Nk, window, page):
    """Grids of uneven sequences that are taken longest first, and the same sequences in another order: same bits."""
    lens = [Nk - 57 * (7 * i % 16) for i in range(16)]
    check_case(16, 8, 2, 330, Nk, D, "bf16", window, 3, lens, page)
    q, k, v = (t.cuda() for t in make_qkv(16, 8, 2, 330, Nk, D, "bf16", seed=5))
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = fa.fwd_window(q, k, v, window, sinks=3, seqlens_k=sl)
    turn = torch.arange(15, -1, -1, device="cuda")
    ot, lt = fa.fwd_window(q[turn].contiguous(), k[turn].contiguous(), v[turn].contiguous(), window, sinks=3, seqlens_k=sl[turn].contiguous())
    assert torch.equal(ot, o[turn]) and torch.equal(lt, lse[turn])


@pytest.mark.parametrize("Hq,Hkv,N,D,dt", [(14, 2, 777, 64, "f32"), (16, 2, 1111, 96, "bf16"), (32, 8, 300, 80, "f16")])
def test_long_windows_of_other_head_sizes(Hq, Hkv, N, D, dt):
    """Windows of most of the keys take the workgroup layouts of causal calls."""
    for window in (N, N * 3 // 4, N * 3 // 4 - 20):
        check_case(1, Hq, Hkv, N, N, D, dt, window, 2, None, 0)
