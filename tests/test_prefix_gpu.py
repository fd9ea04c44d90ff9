"""fwd_prefix and fwd_prefix_paged against the definition in 64 bits on each
sequence's prefix and suffix one after the other.

Keys past a sequence's length hold NaN, and the table's entry for a suffix page
without valid keys is no page.
The tolerance is that of the attention forward (helpers.check_against)."""
import random

import pytest
import torch

import paper_2608_18656_amd as fa
from paper_2608_18656_amd.inputs import DTYPES, make_qkv

from helpers import check_against, default_scale

pytestmark = pytest.mark.gpu


def reference(q, kp, vp, k, v, total, causal, scale):
    """total[b]: keys of the sequence, prefix first (all of it, or its beginning)."""
    B, Nq, Hq, D = q.shape
    Hkv = kp.shape[1]
    o, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full((B, Hq, Nq), -torch.inf, dtype=torch.float64)
    for b in range(B):
        n = total[b]
        K, V = torch.cat([kp, k[b]])[:n].double(), torch.cat([vp, v[b]])[:n].double()
        see = torch.ones((Nq, n), dtype=torch.bool)
        if causal:
            see = torch.arange(n)[None] <= n - Nq + torch.arange(Nq)[:, None]
        rows = see.any(1)
        if not rows.any():
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            x = ((q[b, :, h].double() @ K[:, g].t()) * scale).masked_fill(~see, -torch.inf)[rows]
            lse[b, h, rows] = torch.logsumexp(x, 1)
            o[b, rows, h] = torch.softmax(x, 1) @ V[:, g]
    return o.numpy(), lse.numpy()


def check_case(B, Hq, Hkv, Nq, Np, Nk, D, dt, causal, lens, page, seed=7, scale=None):
    """lens: suffix keys; paged: keys in all, which may be fewer than the prefix's.  None: Nk each."""
    q, k, v = make_qkv(B, Hq, Hkv, Nq, max(Nk, 1), D, dt, seed=seed)
    _, kp, vp = (t[0] if t.shape[0] == 1 else t for t in make_qkv(1, Hq, Hkv, 1, Np, D, dt, seed=seed + 1))
    scale = default_scale(D) if scale is None else scale
    n = lens if lens is not None else [Nk + (Np if page else 0)] * B
    total = [max(0, min(x, Np + Nk)) for x in n] if page else [Np + max(0, min(x, Nk)) for x in n]
    ref = reference(q, kp, vp, k, v, total, causal, scale)
    k, v = k.clone(), v.clone()
    for b in range(B):
        k[b, max(total[b] - Np, 0):] = float("nan")
        v[b, max(total[b] - Np, 0):] = float("nan")
    kw = dict(causal=causal, scale=scale)
    sl = torch.tensor(n, dtype=torch.int32, device="cuda") if lens is not None or page else None
    if page:
        assert Np % page == 0 and Nk % page == 0
        np_, ns = Np // page, Nk // page
        gen = torch.Generator().manual_seed(seed)
        perm = torch.randperm(np_ + B * ns + 1, generator=gen).int()
        pools = []
        for pre, suf in ((kp, k), (vp, v)):
            pool = torch.full((np_ + B * ns + 1, page, Hkv, D), float("nan"), dtype=pre.dtype)
            longest = max(total)   # keys of the prefix that no sequence has
            pre = pre.clone()
            pre[min(longest, Np):] = float("nan")
            pool[perm[:np_].long()] = pre.view(np_, page, Hkv, D)
            if ns:
                pool[perm[np_:-1].long()] = suf.reshape(B * ns, page, Hkv, D)
            pools.append(pool.cuda())
        table = torch.full((B, np_ + ns), 1 << 30, dtype=torch.int32)
        table[:, :np_] = perm[:np_]
        for b in range(B):
            used = -(-max(total[b] - Np, 0) // page)
            table[b, np_:np_ + used] = perm[np_ + b * ns:np_ + b * ns + used]
        table = table.cuda()
        call = lambda odt, **x: fa.fwd_prefix_paged(q.cuda(), *pools, table, sl, Np, out_dtype=odt, **kw, **x)   # noqa: E731
    else:
        call = lambda odt, **x: fa.fwd_prefix(q.cuda(), kp.cuda(), vp.cuda(), k.cuda(), v.cuda(), seqlens_k=sl,   # noqa: E731
                                              out_dtype=odt, **kw, **x)
    for odt in (torch.float32, DTYPES[dt]):
        o, lse = call(odt)
        torch.cuda.synchronize()
        none = torch.isneginf(torch.from_numpy(ref[1]))
        assert torch.equal(torch.isneginf(lse.cpu()), none)
        assert bool((o.cpu().transpose(1, 2)[none] == 0).all())
        ok = torch.where(none, 0.0, lse.cpu().double()), torch.where(none, 0.0, torch.from_numpy(ref[1]))
        check_against(o, ok[0], ref[0], ok[1].numpy(), DTYPES[dt], odt == torch.float32,
                      f"prefix {B, Hq, Hkv, Nq, Np, Nk, D, dt, causal, lens, page, odt}")


EDGES = [
    # one token a sequence
    (4, 32, 4, 1, 2000, 64, 128, "f16", True, [64, 9, 0, 1], 0),
    (3, 8, 2, 1, 1, 1, 64, "bf16", True, [1, 0, 1], 0),
    (2, 16, 1, 1, 33, 5, 64, "f16", False, None, 0),
    (64, 32, 8, 1, 640, 128, 128, "bf16", True, [128 - 2 * i for i in range(64)], 0),
    (9, 40, 8, 1, 1500, 700, 64, "bf16", True, [700 - 80 * i for i in range(9)], 0),
    (5, 4, 4, 1, 5000, 300, 128, "f16", True, [300, 0, 31, 32, 33], 0),
    (6, 32, 8, 1, 1024, 256, 128, "bf16", True, [1280, 1024, 1025, 1000, 0, 64], 64),     # shorter than the prefix, and empty
    (4, 16, 2, 1, 8192, 0, 64, "f16", True, [8192, 1, 8000, 4096], 64),                    # no room for suffixes; more than 64 pages
    (1, 8, 8, 1, 256, 512, 64, "bf16", False, [700], 256),
    # several rows
    (3, 8, 2, 5, 100, 40, 64, "bf16", True, [40, 5, 3], 0),               # a suffix shorter than the new tokens: some are in the prefix
    (3, 8, 2, 70, 50, 100, 128, "f16", True, [100, 30, 0], 0),            # rows before the prefix's first key
    (2, 32, 8, 129, 777, 300, 128, "bf16", True, [300, 200], 0),
    (2, 32, 8, 129, 777, 300, 64, "bf16", False, [300, 0], 0),
    (3, 6, 3, 33, 640, 128, 64, "f16", True, [768, 650, 600], 128),
    (2, 4, 4, 64, 5120, 128, 128, "bf16", True, [5248, 5200], 64),
    (2, 4, 4, 64, 5120, 128, 128, "bf16", False, [5248, 5000], 64),
    (40, 4, 1, 3, 320, 64, 64, "bf16", True, [64 + 320 - 3 * i for i in range(40)], 64),
    (2, 8, 2, 31, 90, 40, 64, "f16", True, [40, 20], 0),                  # one pass: few keys
    (2, 8, 2, 32, 90, 40, 64, "f16", True, [40, 20], 0),
    (2, 8, 2, 32, 2500, 90, 64, "f16", True, [90, 20], 0),                # parts, full waves
    (40, 8, 4, 260, 90, 300, 64, "f16", True, [300 - 7 * i for i in range(40)], 0),    # one pass: full chip
    (24, 8, 8, 300, 200, 320, 128, "bf16", True, [320 - 13 * i for i in range(24)], 0),
    (12, 3, 1, 1, 30, 9, 128, "bf16", True, list(range(10)) + [9, 9], 0),  # one pass, one row
    (12, 16, 1, 1, 64, 64, 64, "bf16", False, [64 + 5 * i for i in range(12)], 64),
    (2, 8, 2, 31, 128, 64, 128, "bf16", True, [192, 100], 64),
    (2, 8, 2, 32, 128, 64, 128, "bf16", True, [192, 100], 64),
    (2, 16, 2, 7, 500, 3, 64, "f16", True, [3, 1], 0),                    # fewer suffix rows than queries
]


@pytest.mark.parametrize("case", EDGES, ids=lambda c: "-".join(str(x) for x in c[:9]) + f"-{c[10]}")
def test_edges(case):
    check_case(*case)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
@pytest.mark.parametrize("Nq,D,dt", [(1, 64, "bf16"), (1, 128, "f16"), (40, 128, "bf16")])
def test_scales(scale, Nq, D, dt):
    check_case(3, 8, 2, Nq, 500, 90, D, dt, True, [90, 50, 41], 0, scale=scale)


def _random_case(seed):
    r = random.Random(seed)
    page = r.choice((0, 0, 64, 128))
    Hkv = r.choice((1, 2, 3, 8))
    Hq, B = Hkv * r.choice((1, 2, 4, 5, 8, 17)), r.randint(1, 9)
    Np, Nk = r.choice((r.randint(1, 100), r.randint(100, 3000))), r.choice((r.randint(1, 40), r.randint(1, 400)))
    if page:
        Np, Nk = page * max(1, Np // page), page * (Nk // page)
    Nq = r.choice((1, 1, r.randint(1, min(Np + Nk, 60))))
    lens = None if not page and r.random() < 0.2 else [r.randint(0, Nk) + (r.choice((Np, Np, Np, 0)) if page else 0) for _ in range(B)]
    return (B, Hq, Hkv, Nq, Np, Nk, r.choice((64, 128)), r.choice(("f16", "bf16")), r.random() < 0.7, lens, page, seed)


@pytest.mark.parametrize("seed", range(40))
def test_random(seed):
    check_case(*_random_case(seed))


def test_equals_the_paged_cache():
    """Against fwd_kvcache_paged on the same cache, within both sides' rounding of the weights (2^-11 of |v| <= 6 each)."""
    B, Hq, Hkv, D, P = 5, 16, 4, 128, 64
    for Nq in (1, 20):
        q = torch.randn((B, Nq, Hq, D), device="cuda").to(torch.bfloat16)
        pool = torch.randn((60, P, Hkv, D), device="cuda").to(torch.bfloat16), torch.randn((60, P, Hkv, D), device="cuda").to(torch.bfloat16)
        own = torch.arange(20, 20 + 5 * B, dtype=torch.int32).view(B, 5)
        table = torch.cat([torch.arange(20, dtype=torch.int32).flip(0).expand(B, 20), own], 1).contiguous().cuda()
        n = torch.tensor([1600, 1281, 1300, 1500, 1320], dtype=torch.int32, device="cuda")
        a, la = fa.fwd_kvcache_paged(q, *pool, table, n, causal=True, out_dtype=torch.float32)
        b, lb = fa.fwd_prefix_paged(q, *pool, table, n, 1280, causal=True, out_dtype=torch.float32)
        assert float((a - b).abs().max()) <= 12 * 2.0 ** -11 and float((la - lb).abs().max()) <= 2.0 ** -10


def test_long_prefix_rows_past_31_bits():
    Np, Hkv, D = 300_000, 64, 128
    kp = torch.zeros((Np, Hkv, D), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    kp[-300:], vp[-300:] = 4 * torch.randn_like(kp[-300:]), torch.randn_like(vp[-300:])
    k, v = torch.randn((2, 5, Hkv, D), device="cuda").to(kp.dtype), torch.randn((2, 5, Hkv, D), device="cuda").to(kp.dtype)
    q = torch.randn((2, 1, Hkv, D), device="cuda").to(kp.dtype)
    o, lse = fa.fwd_prefix(q, kp, vp, k, v, scale=3.0, out_dtype=torch.float32)
    # the zero keys weigh 1 each: a softmax over them, the last 300 and the suffix
    x = 3.0 * torch.einsum("bhd,bkhd->bhk", q[:, 0].double().cpu(), torch.cat([kp[-300:].expand(2, 300, Hkv, D), k], 1).double().cpu())
    ref = torch.logsumexp(torch.cat([x, torch.full((2, Hkv, 1), float(torch.tensor(Np - 300.0).log()), dtype=torch.float64)], 2), 2)
    w = torch.exp(x - ref[..., None])
    r = torch.einsum("bhk,bkhd->bhd", w, torch.cat([vp[-300:].expand(2, 300, Hkv, D), v], 1).double().cpu())
    assert float((lse[:, :, 0].cpu().double() - ref).abs().max()) <= 2e-3
    assert float((o[:, 0].cpu().double() - r).abs().max()) <= 2e-3


def test_workspaces():
    B, Hq, Hkv, Np, Nk, D = 6, 32, 8, 3000, 400, 128
    q, k, v = (t.cuda() for t in make_qkv(B, Hq, Hkv, 1, Nk, D, "bf16", seed=4))
    kp, vp = (t[0].contiguous().cuda() for t in make_qkv(1, Hq, Hkv, 1, Np, D, "bf16", seed=5)[1:])
    need = fa.prefix_workspace_bytes(B, Hq, Hkv, 1, Np, Nk, D, "bf16")
    ref, lse = fa.fwd_prefix(q, kp, vp, k, v)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    mine, mlse = fa.fwd_prefix(q, kp, vp, k, v, workspace=ws)
    assert torch.equal(ref, mine) and torch.equal(lse, mlse)
    with pytest.raises(fa.FaError) as e:
        fa.fwd_prefix(q, kp, vp, k, v, workspace=ws[:4096])
    assert e.value.status == 10
    for Np2, Nk2 in ((1, 1), (100, 400), (2999, 30), (3000, 399), (1500, 200)):   # serves shorter ones
        fa.fwd_prefix(q, kp[:Np2], vp[:Np2], k[:, :Nk2].contiguous(), v[:, :Nk2].contiguous(), workspace=ws)
    torch.cuda.synchronize()
