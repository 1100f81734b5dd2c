"""Cases and plain forms of the operators around a cache that grows: appending
keys and values with the position rotation applied on the way, into caches of the
context's type and into caches held in 4 bits, and attention of newly appended
tokens over a cache held in 4 bits.

``run`` computes a case in elementary torch operations in 32 bits, or, with
``own`` set, through the library's entry points.
"""

import math

import torch

own = False

INF = float("inf")
GROUP = 32  # values that share a scale in a 4-bit cache


# ------------------------------------------------------------------ cases

def _append(name, op, batch, heads, kv_heads, dim, dtype, new, len_lo, len_hi, page, rot, interleaved, axes, ragged):
    c = dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, new=new, len_lo=len_lo,
             len_hi=len_hi, page=page, rot=rot, interleaved=interleaved, axes=axes, ragged=ragged)
    return dict(c, name=name) if name else c


def _attend(name, batch, heads, kv_heads, dim, dtype, new, len_lo, len_hi, page, window, sinks, ragged):
    c = dict(op="attend4", batch=batch, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, new=new, len_lo=len_lo,
             len_hi=len_hi, page=page, window=window, sinks=sinks, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One request of a 7B decoder with visual tokens: positions on three axes, paged cache.  Latency.
        _append("append token B1 paged", "append", 1, 28, 4, 128, "bf16", 1, 3857, 3857, 16, 128, False, 3, False),
        # Batched serving, the same decoder.
        _append("append token B32 paged", "append", 32, 28, 4, 128, "bf16", 1, 2816, 6400, 16, 128, False, 3, False),
        # The whole prompt of one request, visual tokens in its middle.  Bandwidth.
        _append("append prompt B1", "append", 1, 28, 4, 128, "bf16", 3857, 3857, 3857, 0, 128, False, 3, False),
        # Drafted tokens of the fp32 workload's layer, different numbers of them; half of a head is rotated.
        _append("append drafted fp32 B16", "append", 16, 8, 2, 64, "fp32", 5, 301, 704, 0, 32, True, 1, True),
        # Batched serving on a 4-bit cache.
        _append("append4 token B32 paged", "append4", 32, 28, 4, 128, "bf16", 1, 2816, 6400, 16, 128, False, 3, False),
        # Four prompts on a 4-bit cache, odd lengths.
        _append("append4 prompt B4", "append4", 4, 32, 8, 128, "bf16", 2305, 2305, 4609, 0, 128, False, 1, True),
        # Attention over a 4-bit cache.  One request of a 7B decoder.  Latency.
        _attend("token4 B1 paged", 1, 28, 4, 128, "bf16", 1, 3857, 3857, 16, -1, 0, False),
        # Batched serving.
        _attend("token4 B32 paged", 32, 28, 4, 128, "bf16", 1, 2816, 6400, 16, -1, 0, False),
        # The largest sweep.  Bandwidth.
        _attend("token4 B64 largest", 64, 32, 8, 128, "bf16", 1, 17408, 17408, 0, -1, 0, False),
        # Drafted tokens, different numbers of them, ragged lengths.
        _attend("drafted4 B16 paged", 16, 32, 8, 128, "bf16", 5, 2305, 9001, 64, -1, 0, True),
        # A windowed layer of an fp32 model in a long cache.
        _attend("token4 fp32 B8 window", 8, 8, 2, 64, "fp32", 1, 20480, 20480, 0, 4096, 4, False),
        # A chunk of a long prompt: the chunks before it lie in the cache.
        _attend("chunk4 B1", 1, 32, 8, 128, "bf16", 1025, 12289, 12289, 0, -1, 0, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        heads, kv_heads, dim = rng.choice([(8, 2, 64), (28, 4, 128), (32, 8, 128), (16, 16, 64), (8, 1, 128)])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        page = rng.choice([0, 0, 16, 64])
        kind = rng.choice(["append", "append4", "token", "token", "few", "chunk"])
        ragged = rng.random() < 0.4
        if kind in ("append", "append4"):
            new = rng.choice([1, rng.randint(2, 8), _log(rng, 9, 4096)])
            batch = _log(rng, 1, 64 if new <= 8 else 8)
            hi = _log(rng, max(new, 64), max(new, 8192))
            lo = rng.randint(max(new, hi // 4), hi)
            rot = rng.choice([dim, dim, dim // 2, 0])
            axes = rng.choice([1, 1, 3]) if rot else 1
            c = _append(None, kind, batch, heads, kv_heads, dim, dtype, new, lo, hi, page, rot, rng.random() < 0.3, axes,
                        ragged)
        else:
            sinks = rng.choice([0, 1, 4, 16])
            window = rng.choice([-1, -1, _log(rng, 32, 4096)])
            new = {"token": 1, "few": rng.randint(2, 8), "chunk": _log(rng, 9, 2048)}[kind]
            batch = _log(rng, 1, 64 if kind != "chunk" else 4)
            hi = max(new, _log(rng, 64, 20480))
            lo = rng.randint(max(new, hi // 4), hi)
            c = _attend(None, batch, heads, kv_heads, dim, dtype, new, lo, hi, page, window, sinks, ragged)
        if _cost(c) <= top and _scores(c) <= 4e9:
            return c


def _scores(c):
    """Bytes of the scores that the plain form holds."""
    return 4.0 * c["batch"] * c["heads"] * c["new"] * c["len_hi"] if c["op"] == "attend4" else 0.0


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 280)


def _lengths(c):
    """Lengths of the batch's sequences, evenly spread over the case's range in a mixed order."""
    b, lo, hi = c["batch"], c["len_lo"], c["len_hi"]
    return [hi if b == 1 else lo + (hi - lo) * ((i * 7 + 3) % b) // (b - 1) for i in range(b)]


def _news(c):
    """New tokens of the batch's sequences."""
    b, n = c["batch"], c["new"]
    return [n - (i * 5 + 1) % b * n // (2 * b) if c["ragged"] else n for i in range(b)]


def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    d, h, hkv = c["dim"], c["heads"], c["kv_heads"]
    held = d // 2 + 2 * (d // GROUP)  # bytes of a row in 4 bits
    total = flops = 0
    for n_tok, n in zip(_lengths(c), _news(c)):
        if c["op"] == "attend4":
            w, s = c["window"], c["sinks"]
            first = n_tok - n
            rows = n_tok if w < 0 else min(n_tok, min(n_tok, n + w - 1) + min(s, max(0, first + 1 - w)))
            if w < 0:
                seen = n * first + n * (n + 1) // 2
            else:
                seen = sum(min(t + 1, w) + min(s, max(0, t + 1 - w)) for t in range(first, n_tok))
            total += rows * hkv * 2 * held + n * h * (2 * d * esz + 4)
            flops += 4 * d * h * seen
        else:
            total += n * (2 * h * d * esz + 2 * hkv * d * esz + c["axes"] * 4 + c["rot"] * 4)
            total += n * 2 * hkv * (d * esz if c["op"] == "append" else held + d * esz)
            flops += n * (3 * (h + hkv) * c["rot"] + (4 * 2 * hkv * d if c["op"] == "append4" else 0))
    return {"bytes": float(total), "flops": float(flops)}


# ------------------------------------------------------------------ inputs

_handle = {}  # the library context of the current shapes, as a program keeps it from call to call


def _table(gen, b, pages, spare):
    n = b * pages + spare
    return torch.randperm(n, generator=gen, device="cuda")[: b * pages].view(b, pages).to(torch.int32), n


def _positions(c, lengths, news):
    """Positions of the new tokens, [axes, batch, new]: with three axes a span of visual tokens, a grid that
    advances on two of them, lies in the middle of the sequence and takes as many positions as its side."""
    axes, n = c["axes"], c["new"]
    if axes == 1:
        return None
    i = torch.arange(n, device="cuda")
    at = torch.tensor(lengths, device="cuda").view(-1, 1) - torch.tensor(news, device="cuda").view(-1, 1) + i
    side = max(1, math.isqrt(c["len_lo"] // 3))
    start = c["len_lo"] // 4
    k = at - start
    inside = (k >= 0) & (k < side * side)
    text = torch.where(at < start, at, at - side * side + side)
    t = torch.where(inside, start + 0 * k, text)
    y = torch.where(inside, start + k // side, text)
    x = torch.where(inside, start + k % side, text)
    return torch.stack([t, y, x]).clamp(min=0).to(torch.int32).contiguous()


def _sections(c):
    """Rotated pairs of each axis: a quarter for the first, the rest shared."""
    pairs = c["rot"] // 2
    if c["axes"] == 1:
        return [pairs]
    a = pairs // 4
    b = (pairs - a) // 2
    return [a, b, pairs - a - b]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1_000_003 + 29)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    b, h, hkv, d, t, n = c["batch"], c["heads"], c["kv_heads"], c["dim"], c["len_hi"], c["new"]
    lengths, news = _lengths(c), _news(c)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    st = dict(case=dict(c), seq_len=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
              new_len=torch.tensor(news, dtype=torch.int32, device="cuda") if c["ragged"] else None)
    page = c["page"]
    if page:
        st["table"], pool = _table(gen, b, -(-t // page), 3)
        lead, rows = pool, page
    else:
        lead, rows = b, t
    # Queries, keys and values of the new tokens lie in the projection's output, side by side.
    qkv = randn(b, n, h + 2 * hkv, d)
    qkv[:, :, h: h + hkv, 5::16] *= 4.0  # some dimensions of the keys are large
    if c["op"] != "attend4":
        qkv = qkv.to(dt)
        st["q"], st["k"], st["v"] = qkv[:, :, :h], qkv[:, :, h: h + hkv], qkv[:, :, h + hkv:]
        st["q_out"] = torch.zeros(b, n, h, d, dtype=dt, device="cuda")
        st["pos"] = _positions(c, lengths, news)
        if c["rot"]:
            angle = torch.arange(t, device="cuda", dtype=torch.float64).view(-1, 1) * torch.exp(
                torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) * (-2 * math.log(1e6) / c["rot"]))
            st["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
            parts = _sections(c)
            st["axis"] = torch.tensor([a for a, x in enumerate(parts) for _ in range(x)], device="cuda")
        if c["op"] == "append":
            st["kc"], st["vc"] = (randn(lead, hkv, rows, d).to(dt) for _ in range(2))
        else:
            for x in ("kc", "vc"):
                st[x] = torch.randint(0, 256, (lead, hkv, rows, d // 2), generator=gen, device="cuda").to(torch.uint8)
                st[x + "_scale"] = torch.rand(lead, hkv, rows, d // GROUP, generator=gen, device="cuda").half()
            st["k_held"], st["v_held"] = (torch.zeros(b, n, hkv, d, dtype=dt, device="cuda") for _ in range(2))
    else:
        # Keys of one token in 32 point along a direction that the queries share in part; the first
        # token's key along one that all of them share (a sink).
        g = h // hkv
        focus = torch.nn.functional.normalize(randn(b, hkv, 1, d), dim=-1)
        sink = torch.nn.functional.normalize(randn(b, hkv, 1, d), dim=-1)
        beta = 0.3 + 0.5 * torch.rand(b, n, hkv, g, 1, generator=gen, device="cuda")
        q = randn(b, n, hkv, g, d) + math.sqrt(d) * (beta * focus.unsqueeze(1) + 0.8 * sink.unsqueeze(1))
        qkv[:, :, :h] = q.view(b, n, h, d)
        st["q"] = qkv.to(dt)[:, :, :h]
        st["out"] = torch.zeros(b, n, h, d, dtype=dt, device="cuda")
        st["lse"] = torch.zeros(b, n, h, device="cuda")
        for x in ("kc", "vc"):
            st[x] = torch.zeros(lead, hkv, rows, d // 2, dtype=torch.uint8, device="cuda")
            st[x + "_scale"] = torch.zeros(lead, hkv, rows, d // GROUP, dtype=torch.half, device="cuda")
            for i in range(b):
                y = randn(hkv, t, d)
                if x == "kc":
                    y[:, 5::32] += 0.8 * math.sqrt(d) * focus[i]
                    y[:, :1] = math.sqrt(d) * sink[i]
                for to, z in zip((st[x], st[x + "_scale"]), _quantise(y.to(dt).float())):
                    if page:
                        ids = st["table"][i].long()
                        z = torch.nn.functional.pad(z, (0, 0, 0, ids.numel() * page - t))
                        to[ids] = z.view(hkv, -1, page, z.shape[-1]).transpose(0, 1)
                    else:
                        to[i] = z
    if own:
        _open(st)
    return st


def _open(st):
    """The library context of the case's shapes and the descriptors of its tensors."""
    from paper_2605_31457_gb300 import vp
    c = st["case"]
    new = c["new"] if c["op"] == "attend4" else 0
    key = (c["batch"], c["heads"], c["kv_heads"], c["dim"], c["len_hi"], c["dtype"], c["page"], new)
    if key not in _handle:
        for ctx in _handle.values():
            vp.vp_free(ctx)
        _handle.clear()
        ctx = vp.vp_init(vp.make_config(c["batch"], c["heads"], c["kv_heads"], c["dim"], 0, c["len_hi"],
                                        vp.VP_BF16 if c["dtype"] == "bf16" else vp.VP_FP32,
                                        1 if c["page"] else 0, c["page"] or 16))
        if new:
            vp.vp_reserve4(ctx, new)
        _handle[key] = ctx
    st["vp"], st["ctx"] = vp, _handle[key]
    if c["op"] == "append":
        st["ck"], st["cv"] = ((vp.kv_paged(st[x], st["table"]) if c["page"] else vp.kv_contiguous(st[x]))
                              for x in ("kc", "vc"))
    else:
        st["ck"], st["cv"] = ((vp.kv4_paged(st[x], st[x + "_scale"], st["table"]) if c["page"]
                               else vp.kv4_contiguous(st[x], st[x + "_scale"])) for x in ("kc", "vc"))
    st["rq"] = vp.rows(st["q"])
    if c["op"] == "attend4":
        st["ro"] = vp.rows(st["out"])
        st["visible"] = vp.make_visible(window=c["window"], sinks=c["sinks"])
    else:
        st["ro"], st["rk"], st["rv"] = vp.rows(st["q_out"]), vp.rows(st["k"]), vp.rows(st["v"])
        st["rotation"] = vp.make_rotation(st["cos_sin"], interleaved=c["interleaved"], positions=st["pos"],
                                          sections=_sections(c)) if c["rot"] else None
        if c["op"] == "append4":
            st["hk"], st["hv"] = vp.rows(st["k_held"]), vp.rows(st["v_held"])


# ------------------------------------------------------------------ one pass

def run(state):
    st, c = state, state["case"]
    if not own:
        return _plain_attend(st) if c["op"] == "attend4" else _plain_append(st)
    vp = st["vp"]
    if c["op"] == "attend4":
        vp.vp_attend4(st["ctx"], c["batch"], c["new"], st["rq"], st["ck"], st["cv"], st["seq_len"], st["visible"],
                      st["ro"], new_len=st["new_len"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if c["op"] == "append":
        vp.vp_append(st["ctx"], c["batch"], c["new"], st["rq"], st["rk"], st["rv"], st["seq_len"], st["rotation"],
                     st["ro"], st["ck"], st["cv"], new_len=st["new_len"])
    else:
        vp.vp_append4(st["ctx"], c["batch"], c["new"], st["rq"], st["rk"], st["rv"], st["seq_len"], st["rotation"],
                      st["ro"], st["ck"], st["cv"], new_len=st["new_len"], k_held=st["hk"], v_held=st["hv"])
    return _append_outputs(st)


def _append_outputs(st):
    got = {"q": st["q_out"], "k": st["kc"], "v": st["vc"]}
    if st["case"]["op"] == "append4":
        got.update(k_scale=st["kc_scale"], v_scale=st["vc_scale"], k_held=st["k_held"], v_held=st["v_held"])
    return got


def _quantise(x):
    """Values in 4 bits, 32 of them to a scale: codes, two to a byte (the even place in the low half), and scales.
    The scale is the least number of four significant bits that is not below 1/7.5 of the largest magnitude."""
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    step = (((top * (1 / 7.5)).view(torch.int32) + 0xFFFFF) & ~0xFFFFF).view(torch.float32).clamp(2.0 ** -14, 61440.0)
    step = torch.where(top.isnan(), top, step)
    code = (g * step.reciprocal().unsqueeze(-1)).round().clamp(-8, 7).add(8).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), step.half()


def _values(codes, scale):
    """What a 4-bit cache holds."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8.0
    return (code.unflatten(-1, (-1, GROUP)) * scale.float().unsqueeze(-1)).flatten(-2)


def _new_places(st):
    """Which rows of the input are new tokens, [batch, new], and their places in the sequences."""
    c = st["case"]
    i = torch.arange(c["new"], device="cuda").view(1, -1)
    n = st["new_len"].long().view(-1, 1) if c["ragged"] else torch.full((c["batch"], 1), c["new"], device="cuda")
    return i < n, st["seq_len"].long().view(-1, 1) - n + i


def _rotate(st, x, place):
    """Rows [batch, new, heads, dim], rotated by their positions, in 32 bits."""
    c, x = st["case"], x.float()
    rot = c["rot"]
    if not rot:
        return x
    pairs = rot // 2
    pos = place.unsqueeze(0) if st["pos"] is None else st["pos"].long()
    pos = pos.permute(1, 2, 0)[:, :, st["axis"]]                                       # [batch, new, pairs]
    pos = pos.clamp(max=st["cos_sin"].shape[0] - 1)                                    # of rows that are no new tokens
    pair = torch.arange(pairs, device="cuda")
    cos = st["cos_sin"][pos, pair].unsqueeze(2)
    sin = st["cos_sin"][pos, pair + pairs].unsqueeze(2)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :pairs], x[..., pairs:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _put(st, cache, rows, new, place):
    """Rows [batch, new, Hkv, ...] to the new tokens' places in a cache.  Rows that are no new tokens write an
    older token's row back."""
    page = st["case"]["page"]
    at = torch.where(new, place, place - st["case"]["new"])
    b = torch.arange(at.shape[0], device="cuda").view(-1, 1).expand_as(at)
    where = (st["table"].long()[b, at // page], slice(None), at % page) if page else (b, slice(None), at)
    cache[where] = torch.where(new.view(*new.shape, 1, 1), rows, cache[where])


def _plain_append(st):
    c = st["case"]
    dt = st["q"].dtype
    new, place = _new_places(st)
    q, k, v = _rotate(st, st["q"], place).to(dt), _rotate(st, st["k"], place).to(dt), st["v"]
    keep = ~new.view(*new.shape, 1, 1)
    st["q_out"].copy_(torch.where(keep, st["q_out"], q))
    if c["op"] == "append":
        _put(st, st["kc"], k, new, place)
        _put(st, st["vc"], v, new, place)
        return _append_outputs(st)
    (kc, ks), (vc, vs) = _quantise(k.float()), _quantise(v.float())
    _put(st, st["kc"], kc, new, place)
    _put(st, st["kc_scale"], ks, new, place)
    _put(st, st["vc"], vc, new, place)
    _put(st, st["vc_scale"], vs, new, place)
    st["k_held"].copy_(torch.where(keep, st["k_held"], _values(kc, ks).to(dt)))
    st["v_held"].copy_(torch.where(keep, st["v_held"], _values(vc, vs).to(dt)))
    return _append_outputs(st)


def _logical(pool, table, rows):
    """A paged cache as [batch, Hkv, rows, ...]."""
    b, pages = table.shape
    x = pool[table.long()]
    return x.transpose(1, 2).reshape(b, pool.shape[1], pages * pool.shape[2], pool.shape[3])[:, :, :rows]


def _whole(st, x):
    """Cache x in 32 bits, [batch, Hkv, tokens, dim]."""
    c = st["case"]
    codes, scale = st[x], st[x + "_scale"]
    if c["page"]:
        codes, scale = (_logical(y, st["table"], c["len_hi"]) for y in (codes, scale))
    return _values(codes, scale)


def _plain_attend(st):
    c = st["case"]
    b, n, hkv, d, t = c["batch"], c["new"], c["kv_heads"], c["dim"], c["len_hi"]
    g = c["heads"] // hkv
    new, place = _new_places(st)
    pos = torch.arange(t, device="cuda")
    at = place.unsqueeze(-1)
    seen = (pos <= at) & new.unsqueeze(-1)
    if c["window"] >= 0:
        seen &= (pos > at - c["window"]) | (pos < c["sinks"])
    q = st["q"].float().reshape(b, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * g, d)
    z = (q @ _whole(st, "kc").transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(b, hkv, n, g, t)
    z.masked_fill_(~seen.view(b, 1, n, 1, t), -INF)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -INF, torch.zeros_like(top), top)
    z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    z.div_(torch.where(total == 0, torch.ones_like(total), total))
    v = _whole(st, "vc") * (pos < st["seq_len"].view(b, 1)).view(b, 1, t, 1)           # rows past the cache are no tokens
    out = z.view(b, hkv, n * g, t) @ v
    st["out"].copy_(out.view(b, hkv, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, c["heads"], d))
    st["lse"].copy_((total.log() + top).view(b, hkv, n, g).permute(0, 2, 1, 3).reshape(b, n, c["heads"]))
    return {"out": st["out"], "lse": st["lse"]}


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    c = case
    st = prepare(case, seed)
    lengths, news = _lengths(c), _news(c)
    b, n, h, hkv, d, page = c["batch"], c["new"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    if c["op"] != "attend4":
        pairs = c["rot"] // 2

        def turned(x, i):
            """The new tokens' rows of sequence i, rotated as complex numbers, pair by pair."""
            y = x[i, : news[i]].double().clone()
            for p in range(pairs):
                lo, hi = (2 * p, 2 * p + 1) if c["interleaved"] else (p, p + pairs)
                axis, edge = 0, _sections(c)[0]
                while p >= edge:
                    axis += 1
                    edge += _sections(c)[axis]
                at = (st["pos"][axis, i, : news[i]].long() if st["pos"] is not None
                      else torch.arange(lengths[i] - news[i], lengths[i], device="cuda"))
                w = torch.complex(st["cos_sin"][at, p].double(), st["cos_sin"][at, p + pairs].double())
                z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * w.unsqueeze(-1)
                y[..., lo], y[..., hi] = z.real, z.imag
            return y

        q_out = st["q_out"].double()
        kc = st["kc"].double() if c["op"] == "append" else None
        vc = st["vc"].double() if c["op"] == "append" else None
        for i in range(b):
            q_out[i, : news[i]] = turned(st["q"], i)
            if kc is not None:
                at = torch.arange(lengths[i] - news[i], lengths[i], device="cuda")
                where, row = (st["table"][i].long()[at // page], at % page) if page else (torch.full_like(at, i), at)
                kc[where, :, row] = turned(st["k"], i)
                vc[where, :, row] = st["v"][i, : news[i]].double()
        got = {"q": q_out, "k": kc, "v": vc}
        # What is rounded to 4 bits has no value in 64.
        return got if c["op"] == "append" else dict(got, k_scale=None, v_scale=None, k_held=None, v_held=None)
    grp = h // hkv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -INF, dtype=torch.float64, device="cuda")

    def cached(x, i, g, j):
        """Rows j of one (sequence, kv-head) of a cache, in 64 bits."""
        where, row = (st["table"][i].long()[j // page], j % page) if page else (torch.full_like(j, i), j)
        codes = st[x][where, g, row].long()
        y = torch.zeros(j.numel(), d, dtype=torch.float64, device="cuda")
        y[:, 0::2] = (codes % 16 - 8).double()
        y[:, 1::2] = (codes // 16 - 8).double()
        return y * st[x + "_scale"][where, g, row].double().repeat_interleave(GROUP, 1)

    for i in range(b):
        for g in range(hkv):
            heads = slice(g * grp, (g + 1) * grp)
            for q0 in range(0, news[i], 1024):
                q1 = min(news[i], q0 + 1024)
                first, last = lengths[i] - news[i] + q0, lengths[i] - news[i] + q1 - 1
                low = 0 if c["window"] < 0 else max(0, first - c["window"] + 1)
                j = torch.cat([torch.arange(0, min(c["sinks"], low), device="cuda"),
                               torch.arange(low, last + 1, device="cuda")])
                q = st["q"][i, q0:q1, heads].double()
                z = torch.einsum("nhd,jd->nhj", q, cached("kc", i, g, j)) / math.sqrt(d)
                at = torch.arange(first, last + 1, device="cuda").view(-1, 1)
                hidden = j > at
                if c["window"] >= 0:
                    hidden |= (j <= at - c["window"]) & (j >= c["sinks"])
                z = z.masked_fill(hidden.unsqueeze(1), -INF)
                s = torch.logsumexp(z, -1)
                p = torch.exp(z - torch.where(s == -INF, torch.zeros_like(s), s).unsqueeze(-1))
                out[i, q0:q1, heads] = torch.einsum("nhj,jd->nhd", p, cached("vc", i, g, j))
                lse[i, q0:q1, heads] = s
    return {"out": out, "lse": lse}
