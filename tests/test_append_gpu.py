"""kvcache_append and kvcache_append_paged against the definition in 64 bits.

Every written element is compared, every other row of the caches (filled with
NaN patterns of the type) must keep its bits.  Tolerance: sine and cosine are
off by at most 3.4e-7 (the reduced angle's rounding, pi 2^-25, and four units of
2^-24 in the functions), the products and their sum by three
roundings of 2^-24 more: 6e-7 (|a| + |b|) in all; then half a unit in the
last place of the type, 2^-25 for fp16's subnormals.  Values that do not
rotate are copied."""
import pytest
import torch

import paper_2608_18656_amd as fa

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
INT = {"f16": torch.int16, "bf16": torch.int16, "f32": torch.int32}


def rotated(x, pos, inv_freq, pair_axes, interleaved):
    """x [N, H, D] float64, pos [axes, N] -> (rotated, |a| + |b| of each element's pair, 0 where copied)."""
    pairs = inv_freq.numel()
    t = pos.double()[list(pair_axes)].t() * inv_freq.double()          # [N, pairs]
    c, s = t.cos()[:, None], t.sin()[:, None]
    i0 = torch.arange(pairs) * 2 if interleaved else torch.arange(pairs)
    i1 = i0 + (1 if interleaved else pairs)
    y, mag = x.clone(), torch.zeros_like(x)
    a, b = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = a * c - b * s, a * s + b * c
    mag[..., i0] = mag[..., i1] = a.abs() + b.abs()
    return y, mag


def check(got, ref, mag, dtype):
    eps = torch.finfo(dtype).eps / 2
    tol = torch.where(mag > 0, 6e-7 * mag + eps * ref.abs() * (1 + 1e-6) + (2.0 ** -25 if dtype == torch.float16 else 0), 0.0)
    bad = (got.double() - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, worst {float(((got.double() - ref).abs() - tol).max()):.3e}"


def sentinel(shape, dt, device="cuda"):
    """NaNs, each with other bits."""
    n = 1
    for m in shape:
        n *= m
    i = torch.arange(n, device=device) % 100 + 1
    bits = {torch.float16: 0x7E00, torch.bfloat16: 0x7FC0, torch.float32: 0x7FC00000}[dt]
    it = torch.int32 if dt == torch.float32 else torch.int16
    return (i + bits if dt != torch.bfloat16 else i % 30 + bits).to(it).view(dt).view(shape)


# B, N, Hq, Hkv, D, rot, interleaved, axes, dtype, page (0: contiguous), Nk, lengths (the new tokens included)
CASES = [
    (1, 1, 32, 4, 64, 64, False, 1, "f16", 256, 1024, [1000]),
    (1, 1, 8, 8, 128, 0, False, 1, "bf16", 0, 5, [1]),                        # no rotation
    (5, 1, 32, 8, 128, 128, False, 1, "bf16", 64, 640, [640, 1, 65, 0, 641]),  # a sequence without tokens, one past the cache
    (3, 7, 16, 2, 64, 32, False, 1, "bf16", 0, 40, [40, 7, 3]),               # half of the columns, padding
    (2, 9, 6, 3, 80, 80, True, 3, "f16", 0, 33, [33, 12]),
    (2, 33, 16, 1, 128, 128, False, 3, "bf16", 64, 128, [100, 64]),           # a page's edge inside the new tokens
    (2, 5, 4, 2, 40, 40, False, 1, "f16", 0, 8, [8, 6]),                      # halves of 20 columns
    (1, 3, 2, 1, 8, 2, False, 1, "f32", 0, 3, [3]),
    (1, 3, 2, 2, 24, 6, True, 2, "f32", 64, 64, [9]),
    (2, 4, 5, 5, 56, 48, False, 4, "f32", 0, 4, [4, 4]),
    (1, 2, 2, 2, 256, 256, False, 4, "bf16", 0, 2, [2]),
    (2, 777, 8, 8, 72, 24, True, 1, "bf16", 64, 1024, [1000, 777]),            # past the size where four tokens share a workgroup
    (1, 1031, 32, 8, 96, 96, False, 3, "f16", 0, 1200, [1100]),
    (3, 401, 2, 1, 88, 34, True, 1, "f32", 0, 500, [500, 401, 200]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:11]))
@pytest.mark.parametrize("fused", [False, True])
def test_append(case, fused):
    B, N, Hq, Hkv, D, rot, inter, axes, dt, page, Nk, lens = case
    dtype = DT[dt]
    gen = torch.Generator().manual_seed(B * 1000 + N + D)
    W = (Hq + 2 * Hkv) * D
    qkv = (torch.randn(B, N, W, generator=gen) * 2).to(dtype)
    q, k, v = (t.unflatten(2, (-1, D)) for t in qkv.split((Hq * D, Hkv * D, Hkv * D), dim=2))
    dq, dk, dv = (t.unflatten(2, (-1, D)) for t in qkv.cuda().split((Hq * D, Hkv * D, Hkv * D), dim=2))
    if not fused:
        dq, dk, dv = dq.contiguous(), dk.contiguous(), dv.contiguous()
    freq = pos = pair_axes = None
    if rot:
        freq = (1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()
        pair_axes = [j * axes // (rot // 2) for j in range(rot // 2)] if rot // 2 >= axes else [0] * (rot // 2)
        if axes > 1:   # far, negative and near positions
            pos = torch.randint(-50, 1 << 20, (axes, B, N), generator=gen, dtype=torch.int32)
            pos[0, 0, 0] = 2 ** 26 + 1
    lengths = torch.tensor(lens, dtype=torch.int32)
    kw = dict(inv_freq=freq.cuda() if rot else None, positions=pos.cuda() if pos is not None else None,
              pair_axes=bytes(pair_axes) if axes > 1 else None, interleaved=inter)
    if page:
        n = Nk // page
        table = torch.randperm(B * n + 2, generator=gen)[:B * n].view(B, n).int()
        kc, vc = (sentinel((B * n + 2, page, Hkv, D), dtype) for _ in range(2))
        before = kc.clone()
        qo = fa.kvcache_append_paged(dk, dv, kc, vc, table.cuda(), lengths.cuda(), q=dq, **kw)
    else:
        kc, vc = (sentinel((B, Nk, Hkv, D), dtype) for _ in range(2))
        before = kc.clone()
        qo = fa.kvcache_append(dk, dv, kc, vc, lengths.cuda(), q=dq, **kw)
    torch.cuda.synchronize()
    assert qo.shape == q.shape and qo.is_contiguous()
    it = INT[dt]
    kept = torch.ones(kc.shape[:2], dtype=torch.bool)
    kc, vc, qo, before = kc.cpu(), vc.cpu(), qo.cpu(), before.cpu()
    for b in range(B):
        r = torch.arange(lens[b] - N, lens[b])
        p = pos[:, b] if pos is not None else r[None]
        if rot:
            axis = pair_axes if axes > 1 else [0] * (rot // 2)
            kr, km = rotated(k[b].double(), p, freq, axis, inter)
            qr, qm = rotated(q[b].double(), p, freq, axis, inter)
        else:
            kr, km, qr, qm = k[b].double(), torch.zeros(1), q[b].double(), torch.zeros(1)
        check(qo[b], qr, qm, dtype)
        ok = (r >= 0) & (r < Nk)
        if not ok.any():
            continue
        r = r[ok]
        at = (table[b].long()[r // page], r % page) if page else (torch.full_like(r, b), r)
        check(kc[at], kr[ok], km[ok] if rot else km, dtype)
        assert torch.equal(vc[at].view(it), v[b][ok].contiguous().view(it))
        kept[at] = False
    for c in (kc, vc):
        assert torch.equal(c[kept].view(it), before[kept].view(it))


def test_far_rows_of_a_long_cache():
    """Rows past 2^31 elements of the caches."""
    Hkv, D, Nk = 16, 256, 600_000
    kc = torch.zeros((1, Nk, Hkv, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    k = torch.randn((1, 3, Hkv, D), device="cuda").to(torch.bfloat16)
    v = torch.randn((1, 3, Hkv, D), device="cuda").to(torch.bfloat16)
    fa.kvcache_append(k, v, kc, vc, torch.tensor([Nk], dtype=torch.int32, device="cuda"))
    pages = kc.view(-1, 64, Hkv, D), vc.view(-1, 64, Hkv, D)
    table = torch.arange(Nk // 64 - 1, -1, -1, dtype=torch.int32, device="cuda")[None]
    fa.kvcache_append_paged(k + 1, v + 1, *pages, table, torch.tensor([2], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(kc[0, -3:], k[0]) and torch.equal(vc[0, -3:], v[0])
    last = Nk - 64
    assert torch.equal(kc[0, last:last + 2], (k + 1)[0, 1:]) and torch.equal(vc[0, last:last + 2], (v + 1)[0, 1:])
    assert int((kc[0].view(torch.int16).amax((1, 2)) != 0).sum()) == 5


def test_entries_outside_the_pool_are_skipped():
    kc = sentinel((3, 64, 2, 64), torch.float16)
    vc = sentinel((3, 64, 2, 64), torch.float16)
    before = kc.clone()
    table = torch.tensor([[0, -1], [3, 1], [1 << 30, 2]], dtype=torch.int32, device="cuda")
    k = torch.ones((3, 2, 2, 64), dtype=torch.float16, device="cuda")
    fa.kvcache_append_paged(k, k, kc, vc, table, torch.tensor([65, 65, 64], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    kept = torch.ones((3, 64), dtype=torch.bool)
    kept[0, 63] = kept[1, 0] = False   # rows 63 of the first sequence and 64 of the second
    for c in (kc, vc):
        assert torch.equal(c.cpu()[kept].view(torch.int16), before.cpu()[kept].view(torch.int16))
        assert (c.cpu()[~kept] == 1).all()


@pytest.mark.parametrize("inter,rot,D", [(False, 128, 128), (True, 64, 128), (False, 40, 40), (True, 6, 24)])
def test_in_place_and_out(inter, rot, D):
    """q rotated in place, and into a given tensor, as into a new one."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k = (torch.randn((2, 700, h, D), generator=gen, device="cuda").to(torch.bfloat16) for h in (8, 2))
    freq = torch.rand(rot // 2, generator=gen, device="cuda")
    lens = torch.tensor([700, 900], dtype=torch.int32, device="cuda")
    kc, vc = torch.zeros((2, 900, 2, D), dtype=q.dtype, device="cuda"), torch.zeros((2, 900, 2, D), dtype=q.dtype, device="cuda")
    args = dict(inv_freq=freq, interleaved=inter)
    ref = fa.kvcache_append(k, k, kc, vc, lens, q=q, **args)
    kept = kc.clone()
    out = torch.empty_like(q)
    assert fa.kvcache_append(k, k, kc, vc, lens, q=q, q_out=out, **args) is out
    mine = q.clone()
    assert fa.kvcache_append(k, k, kc, vc, lens, q=mine, q_out=mine, **args) is mine
    assert fa.kvcache_append(k, k, kc, vc, lens, **args) is None
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and torch.equal(mine, ref) and torch.equal(kc, kept)


def test_python_refusals():
    k = torch.zeros((2, 3, 2, 64), dtype=torch.float16, device="cuda")
    c = torch.zeros((2, 8, 2, 64), dtype=torch.float16, device="cuda")
    n = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    f = torch.ones(32, device="cuda")
    for bad in (dict(v=k[:, :2]), dict(v=k.float()), dict(k_cache=c[:1]), dict(k_cache=c.bfloat16()), dict(seqlens_k=n.long()),
                dict(seqlens_k=n[:1]), dict(k=k.cpu(), v=k.cpu()), dict(k=k.transpose(1, 2), v=k.transpose(1, 2)),
                dict(k=k[:, :1].expand(2, 3, 2, 64), v=k), dict(q=k.float()), dict(q_out=k), dict(inv_freq=f.double()),
                dict(positions=n.view(2, 1)), dict(inv_freq=f, positions=n.view(2, 1).expand(2, 3)),
                dict(inv_freq=f, positions=torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda")),
                dict(inv_freq=f, positions=torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda"), pair_axes=bytes(31))):
        args = dict(dict(k=k, v=k, k_cache=c, v_cache=c.clone(), seqlens_k=n), **bad)
        with pytest.raises(ValueError):
            fa.kvcache_append(**args)
    for bad, code in ((dict(inv_freq=torch.ones(33, device="cuda")), 14), (dict(v_cache=c), 8),
                      (dict(inv_freq=f, positions=torch.zeros((5, 2, 3), dtype=torch.int32, device="cuda"), pair_axes=bytes(32)), 14),
                      (dict(inv_freq=f, positions=torch.zeros((2, 2, 3), dtype=torch.int32, device="cuda"), pair_axes=bytes([2] * 32)), 14)):
        args = dict(dict(k=k, v=k, k_cache=c, v_cache=c.clone(), seqlens_k=n), **bad)
        with pytest.raises(fa.FaError) as e:
            fa.kvcache_append(**args)
        assert e.value.status == code
