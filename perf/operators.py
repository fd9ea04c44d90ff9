"""The serving operators' measured calls: keys and values appended to a cache with
the position rotation on the way, attention with a sliding window and first
tokens that stay visible, and attention of a batch that shares a long prefix.

A case is a dict with an "op" and the sizes of that operator:
  append  q, k, v of N new tokens a sequence, as views of one fused projection
          [B, N, (Hq + 2 Hkv) D]: q and k rotated by their positions, k and v
          written to the rows that the lengths name, of a contiguous cache or
          of shuffled pages                   (kvcache_append, kvcache_append_paged)
  window  q [B, Nq, Hq, D], each sequence's last Nq positions, against the
          ``window`` keys up to its own and the first ``sinks``  (fwd_window, fwd_window_paged)
  prefix  q [B, Nq, Hq, D] against Np keys that all sequences share and a
          suffix of each sequence's own        (fwd_prefix, fwd_prefix_paged)

Head counts are those of the workloads in paper_2608_18656_amd.inputs (32/4,
32/8, 16/2, 16/16 and 16/1 query / key-value heads).  ``page`` 0 is a contiguous
cache.  Where ``own`` is false, run() is the plain form of the same calls.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = ((32, 4), (32, 8), (16, 2), (16, 16), (16, 1))
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _append(name, dtype, B, Hq, Hkv, N, Nk, D, shortest, page, rot, axes=1, interleaved=False):
    """Lengths, the new tokens included, run evenly from Nk down to ``shortest``; the first ``rot`` columns rotate."""
    return {"name": name, "op": "append", "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "N": N, "Nk": Nk, "D": D,
            "shortest": shortest, "page": page, "rot": rot, "axes": axes, "interleaved": interleaved}


def _window(name, dtype, B, Hq, Hkv, Nq, Nk, D, shortest, page, window, sinks):
    return {"name": name, "op": "window", "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "Nq": Nq, "Nk": Nk, "D": D,
            "shortest": shortest, "page": page, "window": window, "sinks": sinks}


def _prefix(name, dtype, B, Hq, Hkv, Nq, Np, Nk, D, shortest, page):
    """Nk: the longest suffix, which the Nq new tokens end."""
    return {"name": name, "op": "prefix", "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "Nq": Nq, "Np": Np, "Nk": Nk,
            "D": D, "shortest": shortest, "page": page}


def listed():
    return [
        # one user's next token: latency decides
        _append("append_token_f16", "f16", 1, 32, 4, 1, 1537, 64, 1537, 256, 64),
        # a serving step of a large batch, every sequence at its own length
        _append("append_batch_bf16", "bf16", 64, 32, 8, 1, 2048, 128, 300, 64, 128),
        # two long prompts of a larger model, half of each head rotated, in pairs of neighbours
        _append("append_prompt_f16", "f16", 2, 32, 8, 4096, 4096, 128, 4096, 0, 64, 1, True),
        # a prompt with pictures: time, height and width, a number of tokens that divides nothing
        _append("append_axes_bf16", "bf16", 1, 16, 2, 5777, 6144, 128, 5900, 256, 128, 3),
        # one user's next token in a long conversation: latency decides
        _window("window_token_f16", "f16", 1, 32, 8, 1, 8192, 64, 8111, 0, 1024, 4),
        # a serving step of a batch of long conversations on a paged cache
        _window("window_batch_bf16", "bf16", 32, 32, 8, 1, 16384, 128, 3000, 64, 4096, 4),
        # an ordinary prompt of a model with windowed layers
        _window("window_prompt_bf16", "bf16", 1, 32, 8, 4096, 4096, 128, 4096, 0, 1024, 4),
        # a very long prompt on one key/value head
        _window("window_long_f16", "f16", 1, 16, 1, 16384, 16384, 64, 16384, 0, 2048, 64),
        # a chunk of a prompt in full precision, odd sizes, a head size other than 64 and 128
        _window("window_chunk_f32", "f32", 2, 16, 2, 333, 1111, 96, 900, 0, 200, 5),
        # a few answers to one question: latency decides
        _prefix("prefix_few_f16", "f16", 4, 32, 4, 1, 2000, 128, 64, 9, 0),
        # a serving step of a large batch behind one long system prompt
        _prefix("prefix_batch_bf16", "bf16", 64, 32, 8, 1, 8192, 1024, 128, 64, 64),
        # questions of different lengths read in behind that prompt
        _prefix("prefix_chunk_bf16", "bf16", 8, 32, 8, 256, 4096, 512, 128, 256, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("append", "window", "window", "prefix", "prefix"))
    Hq, Hkv = rng.choice(HEADS)
    half = rng.choice(("f16", "bf16"))
    D = rng.choice((64, 128))
    page = rng.choice((0, 64, 256))
    if op == "append":
        dtype = rng.choice((half, half, "f32"))
        N = rng.choice((1, _log_int(rng, 1, 4096)))
        B = max(1, min(_log_int(rng, 1, 64), 8192 // N))
        Nk = N + _log_int(rng, 1, 2048)
        axes = rng.choice((1, 3))
        c = _append("", dtype, B, Hq, Hkv, N, Nk, D, rng.randint(N, Nk), page, rng.choice((D, D // 2)), axes,
                    rng.random() < 0.5)
    elif op == "window":
        kind = rng.choice(("token", "prompt", "chunk", "f32"))
        window, sinks = _log_int(rng, 32, 4096), rng.choice((0, 1, 4, rng.randint(1, 128)))
        if kind == "token":
            B, Nk = _log_int(rng, 1, 32), _log_int(rng, 256, 16384)
            c = _window("", half, B, Hq, Hkv, 1, Nk, D, rng.randint(1, Nk), page, window, sinks)
        elif kind == "prompt":
            N, B = _log_int(rng, 64, 16384), rng.randint(1, 4)
            B = max(1, min(B, int(4e9 / (Hq * N * N))))
            N = min(N, int(math.sqrt(4e9 / (B * Hq))), int(1.6e8 / (B * Hq * D)))
            c = _window("", half, B, Hq, Hkv, N, N, D, N, 0, window, sinks)
        elif kind == "chunk":
            Nk = _log_int(rng, 256, 8192)
            Nq = _log_int(rng, 2, min(512, Nk))
            c = _window("", half, rng.randint(1, 4), Hq, Hkv, Nq, Nk, D, rng.randint(max(Nq, Nk // 4), Nk), page,
                        window, sinks)
        else:
            N = _log_int(rng, 64, 1280)
            c = _window("", "f32", 1, 16, rng.choice((2, 16)), N if rng.random() < 0.7 else 1, N,
                        rng.choice((64, 80, 96, 128)), N, 0, min(window, 1024), sinks)
    else:
        Nk = _log_int(rng, 1, 1024)
        Nq = 1 if rng.random() < 0.6 else _log_int(rng, 1, min(256, Nk))
        B = _log_int(rng, 2, 64)
        B = max(2, min(B, 2048 // Nq))
        Np = _log_int(rng, 200, 8192)
        if Nq > 1:
            Np = min(Np, max(200, int(8.4e6 / (B * Nq))))
        if page:
            Np = max(page, Np // page * page)
        c = _prefix("", half, B, Hq, Hkv, Nq, Np, Nk, D, rng.randint(Nq, Nk), page)
    del c["name"]
    return c


def _lengths(case):
    """Each sequence's keys (append: the new ones included; prefix: those of its own)."""
    B, Nk, lo = case["B"], case["Nk"], case["shortest"]
    if B == 1:
        return [lo]
    return [Nk - (Nk - lo) * b // (B - 1) for b in range(B)]


def _pair_axes(case):
    """Axis of each rotated pair: one, or time, height and width in the shares 2 : 3 : 3."""
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return bytes(pairs)
    t, h = pairs // 4, pairs * 3 // 8
    return bytes([0] * t + [1] * h + [2] * (pairs - t - h))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    op, B, Hq, Hkv, Nk, D, page = (case[n] for n in ("op", "B", "Hq", "Hkv", "Nk", "D", "page"))

    def normal(*shape):
        return torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda").to(dt)

    lengths = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    s = {"op": op, "page": page}
    if op == "append":
        N, rot, axes = case["N"], case["rot"], case["axes"]
        qkv = normal(B, N, (Hq + 2 * Hkv) * D)   # one projection's result
        q, k, v = qkv.split((Hq * D, Hkv * D, Hkv * D), dim=2)
        s["q"], s["k"], s["v"] = q.unflatten(2, (Hq, D)), k.unflatten(2, (Hkv, D)), v.unflatten(2, (Hkv, D))
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)).float()
        s["pair_axes"], s["interleaved"] = _pair_axes(case), case["interleaved"]
        if axes > 1:   # a run of text, then frames of height x width patches
            at = torch.arange(N, device="cuda")
            t = lengths.long()[:, None] - N + at
            s["positions"] = torch.stack([t // 64, t // 64 + at % 64 // 8, t // 64 + at % 8]).int().contiguous()
        else:
            s["positions"] = None
        s["pair_axis_index"] = torch.tensor(list(s["pair_axes"]), device="cuda")
    else:
        s["q"] = normal(B, case["Nq"], Hq, D)
    if op == "window":
        s["window"], s["sinks"] = case["window"], case["sinks"]
    if op == "prefix":
        Np = case["Np"]
        kp, vp = normal(Np, Hkv, D), normal(Np, Hkv, D)
    if not page:
        s["k_cache"], s["v_cache"] = normal(B, Nk, Hkv, D), normal(B, Nk, Hkv, D)
        s["lengths"] = lengths
        if op == "prefix":
            s["k_prefix"], s["v_prefix"] = kp, vp
        return s
    # every sequence's pages scattered over the pool; the prefix's pages are in every sequence's table
    n = -(-Nk // page)
    shared = case["Np"] // page if op == "prefix" else 0
    order = torch.randperm(shared + B * n, generator=gen, device="cuda")
    for name in ("k_cache", "v_cache"):
        s[name] = normal(shared + B * n, page, Hkv, D)
    table = order[shared:].view(B, n)
    if op == "prefix":
        s["k_cache"][order[:shared]] = kp.view(shared, page, Hkv, D)
        s["v_cache"][order[:shared]] = vp.view(shared, page, Hkv, D)
        table = torch.cat([order[:shared].expand(B, shared), table], dim=1)
        s["prefix_len"] = case["Np"]
        lengths = lengths + case["Np"]
    s["table"] = table.to(torch.int32).contiguous()
    s["lengths"] = lengths.to(torch.int32)
    return s


def _run_own(s):
    import paper_2608_18656_amd as fa

    if s["op"] == "append":
        turn = {"inv_freq": s["inv_freq"], "positions": s["positions"], "pair_axes": s["pair_axes"],
                "interleaved": s["interleaved"]}
        if s["page"]:
            q = fa.kvcache_append_paged(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], q=s["q"],
                                        **turn)
        else:
            q = fa.kvcache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["lengths"], q=s["q"], **turn)
        return q, s["k_cache"], s["v_cache"]
    if s["op"] == "window":
        if s["page"]:
            return fa.fwd_window_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["window"],
                                       sinks=s["sinks"])
        return fa.fwd_window(s["q"], s["k_cache"], s["v_cache"], s["window"], sinks=s["sinks"], seqlens_k=s["lengths"])
    if s["page"]:
        return fa.fwd_prefix_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["prefix_len"],
                                   causal=True)
    return fa.fwd_prefix(s["q"], s["k_prefix"], s["v_prefix"], s["k_cache"], s["v_cache"], s["lengths"], causal=True)


# ---- plain forms ----


def _turned(x, cos, sin, interleaved):
    """x [B, N, H, D] in 32 bits, its first columns rotated in pairs: neighbours, or halves."""
    pairs = cos.shape[-1]
    c, s = cos[:, :, None], sin[:, :, None]
    a, b = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])
    a, b = a * c - b * s, a * s + b * c
    r = torch.stack((a, b), dim=-1).flatten(-2) if interleaved else torch.cat((a, b), dim=-1)
    return torch.cat((r, x[..., 2 * pairs:]), dim=-1)


def _plain_append(s):
    q, k, v = s["q"], s["k"], s["v"]
    B, N, Hkv, D = k.shape
    rows = s["lengths"].long()[:, None] - N + torch.arange(N, device=q.device)   # cache rows [B, N]
    at = rows[None] if s["positions"] is None else s["positions"]
    # angles of far positions in 64 bits
    angle = at.double().permute(1, 2, 0)[..., s["pair_axis_index"]] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    kr = _turned(k.float(), cos, sin, s["interleaved"]).to(k.dtype)
    qr = _turned(q.float(), cos, sin, s["interleaved"]).to(q.dtype)
    if s["page"]:
        P = s["page"]
        flat = s["table"].long().gather(1, rows // P) * P + rows % P
    else:
        flat = rows + torch.arange(B, device=q.device)[:, None] * s["k_cache"].shape[1]
    s["k_cache"].view(-1, Hkv, D)[flat.view(-1)] = kr.view(-1, Hkv, D)
    s["v_cache"].view(-1, Hkv, D)[flat.view(-1)] = v.reshape(-1, Hkv, D)
    return qr, s["k_cache"], s["v_cache"]


def _grouped(q, Hkv):
    """[B, Nq, Hq, D] -> [B, Hkv, G Nq, D] in 32 bits: a key/value head's rows together."""
    B, Nq, Hq, D = q.shape
    return q.float().view(B, Nq, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)


def _results(o, lse, q):
    """[B, Hkv, G Nq, D] and [B, Hkv, G Nq, 1] as out [B, Nq, Hq, D] and lse [B, Hq, Nq]."""
    B, Nq, Hq, D = q.shape
    return o.reshape(B, Hq, Nq, D).transpose(1, 2).to(q.dtype).contiguous(), lse.reshape(B, Hq, Nq)


def _plain_window(s):
    q, lengths, W, S = s["q"], s["lengths"].long(), s["window"], s["sinks"]
    B, Nq, Hq, D = q.shape
    at = lengths[:, None] - Nq + torch.arange(Nq, device=q.device)   # positions [B, Nq]
    k, v = s["k_cache"], s["v_cache"]
    Hkv, P = k.shape[2], s["page"]
    Nk = s["table"].shape[1] * P if P else k.shape[1]
    if Nq == 1:   # the keys that the row sees, gathered
        j = torch.arange(S + W, device=q.device)
        keys = torch.where(j < S, j, lengths[:, None] - W + j - S)                   # [B, S + W]
        seen = torch.where(j < S, keys < lengths[:, None], keys >= S)[:, None]       # [B, 1, S + W]
        keys = keys.clamp(0, Nk - 1)
    else:
        keys = torch.arange(Nk, device=q.device).expand(B, Nk)
        d = at[:, :, None] - keys[:, None]                                           # [B, Nq, Nk]
        seen = (d >= 0) & ((d < W) | (keys[:, None] < S))
    if P:
        flat = s["table"].long().gather(1, keys // P) * P + keys % P
    else:
        flat = keys + torch.arange(B, device=q.device)[:, None] * Nk
    k = k.view(-1, Hkv, D)[flat].transpose(1, 2).float()                             # [B, Hkv, keys, D]
    v = v.view(-1, Hkv, D)[flat].transpose(1, 2).float()
    x = _grouped(q, Hkv) @ k.transpose(2, 3).contiguous()
    x = x.mul_(1.0 / math.sqrt(D)).view(B, Hkv, Hq // Hkv, Nq, -1)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    x = x.view(B, Hkv, Hq // Hkv * Nq, -1)
    m = x.amax(-1, keepdim=True).clamp_min_(-1e30)
    x = x.sub_(m).exp_()
    n = x.sum(-1, keepdim=True)
    return _results((x @ v.contiguous()) / n, m + n.log(), q)


def _plain_prefix(s):
    q, lengths = s["q"], s["lengths"].long()
    B, Nq, Hq, D = q.shape
    k, v, P = s["k_cache"], s["v_cache"], s["page"]
    Hkv = k.shape[2]
    if P:   # the suffixes' pages and the prefix's
        n, table = s["prefix_len"] // P, s["table"].long()
        kp, vp = k[table[0, :n]].view(-1, Hkv, D), v[table[0, :n]].view(-1, Hkv, D)
        k, v = k[table[:, n:]].view(B, -1, Hkv, D), v[table[:, n:]].view(B, -1, Hkv, D)
        lengths = lengths - s["prefix_len"]
    else:
        kp, vp = s["k_prefix"], s["v_prefix"]
    Np, Nk = kp.shape[0], k.shape[1]
    qg, scale = _grouped(q, Hkv), 1.0 / math.sqrt(D)
    # against the prefix, every sequence's rows of a key/value head together
    rows = qg.transpose(0, 1).reshape(Hkv, -1, D)
    x = (rows @ kp.permute(1, 2, 0).float().contiguous()).mul_(scale)                # [Hkv, B G Nq, Np]
    # against the suffixes
    y = (qg @ k.permute(0, 2, 3, 1).float().contiguous()).mul_(scale)                # [B, Hkv, G Nq, Nk]
    at = lengths[:, None] - Nq + torch.arange(Nq, device=q.device)
    hidden = torch.arange(Nk, device=q.device) > at[:, :, None]                      # [B, Nq, Nk]
    y = y.view(B, Hkv, -1, Nq, Nk).masked_fill_(hidden[:, None, None], -math.inf).reshape(B, Hkv, -1, Nk)
    back = lambda t: t.view(Hkv, B, -1, t.shape[-1]).transpose(0, 1)   # noqa: E731
    m = torch.maximum(back(x.amax(-1, keepdim=True)), y.amax(-1, keepdim=True))
    x = x.sub_(m.transpose(0, 1).reshape(Hkv, -1, 1)).exp_()
    y = y.sub_(m).exp_()
    n = back(x.sum(-1, keepdim=True)) + y.sum(-1, keepdim=True)
    o = back(x @ vp.transpose(0, 1).float().contiguous()) + y @ v.transpose(1, 2).float().contiguous()
    return _results(o / n, m + n.log(), q)


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "window": _plain_window, "prefix": _plain_prefix}[state["op"]](state)


# ---- what the calls cannot do without ----


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    op, B, Hq, Hkv, D = (case[n] for n in ("op", "B", "Hq", "Hkv", "D"))
    lengths = _lengths(case)
    if op == "append":
        tokens = B * case["N"]
        return {"bytes": 2 * tokens * (Hq + 2 * Hkv) * D * e + (4 * case["axes"] * tokens if case["axes"] > 1 else 0),
                "flops": 3 * tokens * (Hq + Hkv) * case["rot"]}
    Nq = case["Nq"]
    if op == "window":
        W, S = case["window"], case["sinks"]
        pairs = keys = 0
        for n in lengths:
            for p in range(n - Nq, n):
                near = min(p + 1, W)
                pairs += near + min(S, p + 1 - near)
            first = max(0, n - Nq + 1 - W)
            keys += n - first + min(S, first)
    else:
        keys = case["Np"] + sum(lengths)
        pairs = sum(Nq * (case["Np"] + n) - Nq * (Nq - 1) // 2 for n in lengths)
    return {"bytes": 2 * B * Nq * Hq * D * e + 4 * B * Hq * Nq + 2 * keys * Hkv * D * e, "flops": 4 * Hq * D * pairs}


# ---- the definitions in 64 bits ----


def _exact_append(case, s):
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    B, N, page, pairs = case["B"], case["N"], case["page"], case["rot"] // 2
    freq, axis = s["inv_freq"].double(), s["pair_axis_index"]
    q_out = s["q"].double()
    for b, n in enumerate(_lengths(case)):
        row = torch.arange(n - N, n, device=freq.device)
        where = row[None] if s["positions"] is None else s["positions"][:, b]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=freq.device), where.double()[axis].t() * freq)
        new_k = s["k"][b].double()
        for t in (new_k, q_out[b]):
            if case["interleaved"]:
                first, second = slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)
            else:
                first, second = slice(0, pairs), slice(pairs, 2 * pairs)
            z = torch.complex(t[..., first].contiguous(), t[..., second].contiguous()) * turn[:, None]
            t[..., first], t[..., second] = z.real, z.imag
        if page:
            to = s["table"][b].long()[row // page], row % page
        else:
            to = torch.full_like(row, b), row
        k_cache[to], v_cache[to] = new_k, s["v"][b].double()
    return q_out, k_cache, v_cache


def _exact_rows(q, k, v, at, where, window, sinks):
    """One sequence: q [Nq, Hq, D] at positions ``at``, k and v [n, Hkv, D] at positions ``where``."""
    Nq, Hq, D = q.shape
    Hkv = k.shape[1]
    o = torch.zeros((Nq, Hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((Hq, Nq), -math.inf, dtype=torch.float64, device=q.device)
    for g in range(Hkv):
        kg, vg = k[:, g].double().t().contiguous(), v[:, g].double().contiguous()
        for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
            for i in range(0, Nq, 4096):
                x = (q[i:i + 4096, h].double() @ kg) / math.sqrt(D)
                d = at[i:i + 4096, None] - where
                x = torch.where((d >= 0) & ((d < window) | (where < sinks)), x, -math.inf)
                lse[h, i:i + 4096] = torch.logsumexp(x, 1)
                o[i:i + 4096, h] = torch.exp(x - lse[h, i:i + 4096, None]) @ vg
    return o, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, s)
    Nq, page, Np = case["Nq"], case["page"], case.get("Np", 0)
    far = 1 << 60
    rows = []
    for b, n in enumerate(_lengths(case)):
        n += Np
        if page:
            pages = s["table"][b].long()
            k, v = (s[c][pages].flatten(0, 1)[:n] for c in ("k_cache", "v_cache"))
        elif Np:
            k, v = (torch.cat((s[p], s[c][b]))[:n] for p, c in (("k_prefix", "k_cache"), ("v_prefix", "v_cache")))
        else:
            k, v = s["k_cache"][b, :n], s["v_cache"][b, :n]
        where = torch.arange(n, device=k.device)
        at = where[n - Nq:]
        if Nq == 1 and "window" in case:   # only what the row may see
            some = torch.cat((where[:case["sinks"]], where[max(case["sinks"], n - case["window"]):]))
            k, v, where = k[some], v[some], some
        rows.append(_exact_rows(s["q"][b], k, v, at, where, case.get("window", far), case.get("sinks", 0)))
    return tuple(torch.stack(t) for t in zip(*rows))
