"""Cases and plain forms of the cache operators: attention of newly appended
tokens over a key-value cache (one token, a few drafted tokens, whole prompts;
sliding window and sink tokens; accumulated attention weights) and eviction
from a cache by accumulated attention weight.

``run`` computes a case in elementary torch operations in 32 bits, or, with
``own`` set, through the library's entry points.
"""

import math

import numpy as np
import torch

own = False

INF = float("inf")


# ------------------------------------------------------------------ cases

def _attend(name, batch, heads, kv_heads, dim, dtype, new, len_lo, len_hi, page, window, sinks, weights):
    c = dict(op="attend", batch=batch, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, new=new,
             len_lo=len_lo, len_hi=len_hi, page=page, window=window, sinks=sinks, weights=weights)
    return dict(c, name=name) if name else c


def _evict(name, batch, kv_heads, dim, dtype, len_lo, len_hi, page, keep, sinks, recent):
    c = dict(op="evict", batch=batch, kv_heads=kv_heads, dim=dim, dtype=dtype, len_lo=len_lo, len_hi=len_hi,
             page=page, keep=keep, sinks=sinks, recent=recent)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The reference workload's layer: one fp32 sequence of 576 visual and 128 text tokens.  Latency.
        _attend("token fp32 B1", 1, 8, 2, 64, "fp32", 1, 704, 704, 0, -1, 0, False),
        # One request of a 7B decoder, paged cache of 1296 visual and 2561 text tokens.  Latency.
        _attend("token B1 paged", 1, 28, 4, 128, "bf16", 1, 3857, 3857, 16, -1, 0, False),
        # Batched serving: 2304 visual and 512 to 4096 text tokens, pages of 16; weights kept for eviction.
        _attend("token B32 paged weights", 32, 28, 4, 128, "bf16", 1, 2816, 6400, 16, -1, 0, True),
        # Long reasoning, 4096 visual and 16384 text tokens, weights kept for eviction.
        _attend("token B8 long weights", 8, 28, 4, 128, "bf16", 1, 20480, 20480, 0, -1, 0, True),
        # A windowed layer of the same decoder: a short visible set in a long cache.
        _attend("token B8 long window", 8, 28, 4, 128, "bf16", 1, 20480, 20480, 0, 4096, 4, False),
        # The largest sweep: 64 sequences of 16384 visual and 1024 text tokens.  Bandwidth.
        _attend("token B64 largest", 64, 32, 8, 128, "bf16", 1, 17408, 17408, 0, -1, 0, False),
        # Four drafted tokens and the current one, ragged lengths.
        _attend("drafted B16 paged", 16, 32, 8, 128, "bf16", 5, 2305, 9001, 64, -1, 0, False),
        # The whole prompt of one request: causal attention, an odd length.
        _attend("prompt B1", 1, 28, 4, 128, "bf16", 3857, 3857, 3857, 0, -1, 0, False),
        # A long prompt through a windowed layer.
        _attend("prompt B1 long window", 1, 32, 8, 128, "bf16", 12289, 12289, 12289, 0, 2048, 4, False),
        # Eviction of one request's cache to about half.  Latency.
        _evict("evict B1 paged", 1, 4, 128, "bf16", 3857, 3857, 16, 2048, 4, 256),
        # Eviction across a serving batch: some sequences are still below the budget.
        _evict("evict B32 paged", 32, 4, 128, "bf16", 2816, 6400, 16, 4096, 4, 512),
        # Long reasoning cut to a fifth.
        _evict("evict B8 long", 8, 4, 128, "bf16", 20480, 20480, 0, 4097, 4, 1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        heads, kv_heads, dim = rng.choice([(8, 2, 64), (28, 4, 128), (32, 8, 128), (16, 16, 64), (8, 1, 128)])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        page = rng.choice([0, 0, 16, 64])
        batch = _log(rng, 1, 64)
        hi = _log(rng, 64, 20480)
        lo = rng.randint(max(1, hi // 4), hi)
        kind = rng.choice(["token", "token", "few", "prompt", "evict", "evict"])
        sinks = rng.choice([0, 1, 4, 16])
        window = rng.choice([-1, -1, _log(rng, 32, 4096)])
        if kind == "token":
            c = _attend(None, batch, heads, kv_heads, dim, dtype, 1, lo, hi, page, window, sinks, rng.random() < 0.5)
        elif kind == "few":
            new = rng.randint(2, 8)
            c = _attend(None, batch, heads, kv_heads, dim, dtype, new, max(lo, new), max(hi, new), page, window, sinks,
                        rng.random() < 0.3)
        elif kind == "prompt":
            new = rng.randint(max(32, hi // 3), max(33, hi))
            hi = max(hi, new)
            c = _attend(None, _log(rng, 1, 8), heads, kv_heads, dim, "bf16", new, hi, hi, page, window, sinks, False)
        else:
            recent = rng.randint(1, max(1, hi // 8))
            keep = rng.randint(sinks + recent, max(sinks + recent, hi - 1))
            c = _evict(None, batch, kv_heads, dim, dtype, lo, hi, page, keep, sinks, recent)
        if _cost(c) <= top and _plain_bytes(c) <= 24e9:
            return c


def _plain_bytes(c):
    """Bytes of the scores that the plain form holds."""
    return 4.0 * c["batch"] * c["heads"] * c["new"] * c["len_hi"] if c["op"] == "attend" else 0.0


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 280)


def _lengths(c):
    """Lengths of the batch's sequences, evenly spread over the case's range in a mixed order."""
    b, lo, hi = c["batch"], c["len_lo"], c["len_hi"]
    return [hi if b == 1 else lo + (hi - lo) * ((i * 7 + 3) % b) // (b - 1) for i in range(b)]


def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    d, hkv = c["dim"], c["kv_heads"]
    total = flops = 0
    for n_tok in _lengths(c):
        if c["op"] == "attend":
            n, w, s = c["new"], c["window"], c["sinks"]
            first = n_tok - n                     # position of the first new token
            rows = n_tok if w < 0 else min(n_tok, min(n_tok, n + w - 1) + min(s, max(0, first + 1 - w)))
            if w < 0:
                seen = n * first + n * (n + 1) // 2
            else:
                seen = sum(min(t + 1, w) + min(s, max(0, t + 1 - w)) for t in range(first, n_tok))
            total += rows * hkv * 2 * d * esz + n * c["heads"] * (2 * d * esz + 4)
            total += 8 * n_tok * hkv if c["weights"] else 0
            flops += 4 * d * c["heads"] * seen
        else:
            k = min(n_tok, c["keep"])
            total += hkv * (4 * n_tok + 8 * k + 4 * d * esz * k)
    return {"bytes": float(total), "flops": float(flops)}


# ------------------------------------------------------------------ inputs

_handle = {}  # the library context of the current shapes, as a program keeps it from call to call


def _table(gen, b, pages, spare):
    n = b * pages + spare
    return torch.randperm(n, generator=gen, device="cuda")[: b * pages].view(b, pages).to(torch.int32), n


def _cache(x, gen, page, cap):
    """A cache of `cap` rows holding x [B, Hkv, T, D]: as it is, or scattered over a pool of shuffled pages."""
    if not page:
        return x, None
    b, h, t, d = x.shape
    pages = -(-cap // page)
    table, n = _table(gen, b, pages, 3)
    pool = torch.zeros(n, h, page, d, dtype=x.dtype, device="cuda")
    x = torch.nn.functional.pad(x, (0, 0, 0, pages * page - t))
    pool[table.long().view(-1)] = x.view(b, h, pages, page, d).transpose(1, 2).reshape(b * pages, h, page, d)
    return pool, table


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1_000_003 + 17)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    b, hkv, d, t = c["batch"], c["kv_heads"], c["dim"], c["len_hi"]

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    st = dict(case=dict(c), seq_len=torch.tensor(_lengths(c), dtype=torch.int32, device="cuda"))
    # Accumulated weights: a few heavy tokens, many light ones, some that were never seen (exactly 0).
    weight = randn(b, hkv, t).mul_(2.0).exp_()
    weight *= torch.rand(b, hkv, t, generator=gen, device="cuda") > 0.15
    k = randn(b, hkv, t, d)
    v = randn(b, hkv, t, d).to(dt)
    if c["op"] == "attend":
        # Keys of one token in 32 point along a direction that the queries share in part; the first
        # token's key along one that all of them share (a sink).
        g, n = c["heads"] // hkv, c["new"]
        focus = torch.nn.functional.normalize(randn(b, hkv, 1, d), dim=-1)
        sink = torch.nn.functional.normalize(randn(b, hkv, 1, d), dim=-1)
        k[:, :, 5::32] += 0.8 * math.sqrt(d) * focus
        k[:, :, :1] = math.sqrt(d) * sink
        beta = 0.3 + 0.5 * torch.rand(b, n, hkv, g, 1, generator=gen, device="cuda")
        q = randn(b, n, hkv, g, d) + math.sqrt(d) * (beta * focus.unsqueeze(1) + 0.8 * sink.unsqueeze(1))
        # The queries lie in the projection's output, next to this step's keys and values.
        qkv = torch.zeros(b, n, c["heads"] + 2 * hkv, d, dtype=dt, device="cuda")
        qkv[:, :, : c["heads"]] = q.view(b, n, c["heads"], d).to(dt)
        st["q"] = qkv[:, :, : c["heads"]]
        st["out"] = torch.zeros(b, n, c["heads"], d, dtype=dt, device="cuda")
        st["lse"] = torch.zeros(b, n, c["heads"], device="cuda")
        st["weight_in"] = weight if c["weights"] else None
        st["weight_out"] = torch.zeros_like(weight) if c["weights"] else None
    else:
        keep, page = c["keep"], c["page"]
        rows = min(keep, t)
        st["weight_in"] = weight
        st["weight_out"] = torch.zeros(b, hkv, rows, device="cuda")
        st["kept"] = torch.zeros(b, hkv, keep, dtype=torch.int32, device="cuda")
        st["count"] = torch.zeros(b, dtype=torch.int32, device="cuda")
        zero = torch.zeros(b, hkv, rows, d, dtype=dt, device="cuda")
        st["k_dst"], st["dst_table"] = _cache(zero, gen, page, rows)
        st["v_dst"] = torch.zeros_like(st["k_dst"])
    st["k"], st["table"] = _cache(k.to(dt), gen, c["page"], t)
    del k
    if c["page"]:
        pool = torch.zeros_like(st["k"])
        x = torch.nn.functional.pad(v, (0, 0, 0, st["table"].shape[1] * c["page"] - t))
        pool[st["table"].long().view(-1)] = (
            x.view(b, hkv, -1, c["page"], d).transpose(1, 2).reshape(-1, hkv, c["page"], d))
        st["v"] = pool
    else:
        st["v"] = v
    if own:
        _open(st)
    return st


def _open(st):
    """The library context of the case's shapes and the descriptors of its tensors."""
    from paper_2605_31457_gb300 import vp
    c = st["case"]
    heads = c.get("heads", c["kv_heads"])
    new, weigh = c.get("new", 0), c.get("weights", False)
    key = (c["batch"], heads, c["kv_heads"], c["dim"], c["len_hi"], c["dtype"], c["page"], new, weigh)
    if key not in _handle:
        for ctx in _handle.values():
            vp.vp_free(ctx)
        _handle.clear()
        ctx = vp.vp_init(vp.make_config(c["batch"], heads, c["kv_heads"], c["dim"], 0, c["len_hi"],
                                        vp.VP_BF16 if c["dtype"] == "bf16" else vp.VP_FP32,
                                        1 if c["page"] else 0, c["page"] or 16))
        if new:
            vp.vp_reserve_new(ctx, new, new if weigh else 0)
        _handle[key] = ctx
    st["vp"], st["ctx"] = vp, _handle[key]
    st["kc"], st["vc"] = ((vp.kv_paged(st[x], st["table"]) if c["page"] else vp.kv_contiguous(st[x])) for x in ("k", "v"))
    st["w_in"] = vp.token_weights(st["weight_in"]) if st["weight_in"] is not None else None
    st["w_out"] = vp.token_weights(st["weight_out"]) if st["weight_out"] is not None else None
    if c["op"] == "attend":
        st["rq"], st["ro"] = vp.rows(st["q"]), vp.rows(st["out"])
        st["visible"] = vp.make_visible(window=c["window"], sinks=c["sinks"])
    else:
        st["kd"], st["vd"] = ((vp.kv_paged(st[x], st["dst_table"]) if c["page"] else vp.kv_contiguous(st[x]))
                              for x in ("k_dst", "v_dst"))
        st["policy"] = vp.make_evict(keep=c["keep"], sinks=c["sinks"], recent=c["recent"], granularity=1)


# ------------------------------------------------------------------ one pass

def run(state):
    c = state["case"]
    if own:
        vp = state["vp"]
        if c["op"] == "attend":
            vp.vp_attend_new(state["ctx"], c["batch"], c["new"], state["rq"], state["kc"], state["vc"],
                             state["seq_len"], state["visible"], state["ro"], lse=state["lse"],
                             weight_in=state["w_in"], weight_out=state["w_out"])
            return _attend_outputs(state)
        vp.vp_evict(state["ctx"], c["batch"], state["kc"], state["vc"], state["seq_len"], state["policy"],
                    state["kd"], state["vd"], state["w_in"], state["w_out"], state["kept"], c["keep"], state["count"])
        return _evict_outputs(state)
    return _plain_attend(state) if c["op"] == "attend" else _plain_evict(state)


def _attend_outputs(st):
    got = {"out": st["out"], "lse": st["lse"]}
    return dict(got, weight=st["weight_out"]) if st["weight_out"] is not None else got


def _evict_outputs(st):
    return {"k": st["k_dst"], "v": st["v_dst"], "weight": st["weight_out"], "kept": st["kept"], "count": st["count"]}


def _logical(pool, table, rows):
    """A paged cache as [B, Hkv, rows, D]."""
    b, pages = table.shape
    x = pool[table.long()]  # [B, pages, Hkv, page, D]
    return x.transpose(1, 2).reshape(b, pool.shape[1], pages * pool.shape[2], pool.shape[3])[:, :, :rows]


def _plain_attend(st):
    c = st["case"]
    b, n, hkv, d, t = c["batch"], c["new"], c["kv_heads"], c["dim"], c["len_hi"]
    g = c["heads"] // hkv
    k, v = (st[x] if not c["page"] else _logical(st[x], st["table"], t) for x in ("k", "v"))
    k, v = k.float(), v.float()
    pos = torch.arange(t, device="cuda")
    at = st["seq_len"].long().view(b, 1) - n + torch.arange(n, device="cuda")     # [B, n] positions of the new tokens
    seen = pos <= at.unsqueeze(-1)
    if c["window"] >= 0:
        seen &= (pos > at.unsqueeze(-1) - c["window"]) | (pos < c["sinks"])
    seen = seen.view(b, 1, n, 1, t)
    v = v * (pos < st["seq_len"].view(b, 1)).view(b, 1, t, 1)                      # rows past the cache are no tokens
    q = st["q"].float().reshape(b, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * g, d)
    z = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(d)).view(b, hkv, n, g, t)
    z.masked_fill_(~seen, -INF)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -INF, torch.zeros_like(top), top)
    z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    z.div_(torch.where(total == 0, torch.ones_like(total), total))
    out = z.view(b, hkv, n * g, t) @ v
    st["out"].copy_(out.view(b, hkv, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, c["heads"], d))
    st["lse"].copy_((total.log() + top).view(b, hkv, n, g).permute(0, 2, 1, 3).reshape(b, n, c["heads"]))
    if c["weights"]:
        live = pos < st["seq_len"].view(b, 1)
        st["weight_out"].copy_(torch.where(live.view(b, 1, t), st["weight_in"] + z.sum((2, 3)), 0.0))
    return _attend_outputs(st)


def _plain_evict(st):
    c = st["case"]
    b, hkv, d, t, keep = c["batch"], c["kv_heads"], c["dim"], c["len_hi"], c["keep"]
    pos = torch.arange(t, device="cuda")
    length = st["seq_len"].long().view(b, 1, 1)
    key = st["weight_in"].masked_fill((pos < c["sinks"]) | (pos >= length - c["recent"]), INF)
    key = key.masked_fill(pos >= length, -INF)
    rows = min(keep, t)
    order = key.sort(dim=-1, descending=True, stable=True).indices[..., :rows]
    count = length.clamp(max=rows)
    slot = torch.arange(rows, device="cuda")
    used = (slot < count).expand(b, hkv, rows)
    kept = order.masked_fill(~used, t).sort(dim=-1).values
    src = kept.clamp(max=t - 1)
    st["kept"].fill_(-1)
    st["kept"][..., :rows] = torch.where(used, kept, -1).to(torch.int32)
    st["count"].copy_(count.view(b))
    st["weight_out"].copy_(st["weight_in"].gather(2, src) * used)
    page = c["page"]
    at = src.unsqueeze(-1).expand(b, hkv, rows, d)
    k, v = (st[x] if not page else _logical(st[x], st["table"], t) for x in ("k", "v"))
    k = k.gather(2, at).masked_fill(~used.unsqueeze(-1), 0.0)
    v = v.gather(2, at).masked_fill(~used.unsqueeze(-1), 0.0)
    if page:
        table = st["dst_table"].long()
        tail = table.shape[1] * page - rows
        k, v = (torch.nn.functional.pad(x, (0, 0, 0, tail)).view(b, hkv, -1, page, d).transpose(1, 2)
                .reshape(-1, hkv, page, d) for x in (k, v))
        st["k_dst"][table.view(-1)] = k
        st["v_dst"][table.view(-1)] = v
    else:
        st["k_dst"].copy_(k)
        st["v_dst"].copy_(v)
    return _evict_outputs(st)


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    c = case
    st = prepare(case, seed)
    lengths = _lengths(c)
    hkv, d = c["kv_heads"], c["dim"]

    def cached(name, i, g, j):
        """Rows j of one (sequence, kv-head) of a cache, in 64 bits."""
        x = st[name]
        if c["page"]:
            ids = st["table"][i].long()
            return x[ids[j // c["page"]], g, j % c["page"]].double()
        return x[i, g, j].double()

    if c["op"] == "evict":
        moved = torch.zeros(st["weight_out"].shape, dtype=torch.float64)
        weight = st["weight_in"].cpu().numpy()
        for i, length in enumerate(lengths):
            for g in range(hkv):
                middle = weight[i, g, c["sinks"]: length - c["recent"]]
                room = c["keep"] - c["sinks"] - c["recent"]
                best = np.sort(np.lexsort((np.arange(middle.size), -middle))[:room]) + c["sinks"]
                rows = np.arange(length) if length <= c["keep"] else np.concatenate(
                    [np.arange(c["sinks"]), best, np.arange(length - c["recent"], length)])
                moved[i, g, : rows.size] = torch.from_numpy(weight[i, g, rows].astype(np.float64))
        return {"k": None, "v": None, "weight": moved, "kept": None, "count": None}
    n, grp = c["new"], c["heads"] // hkv
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -INF, dtype=torch.float64, device="cuda")
    weight = None
    if c["weights"]:
        weight = torch.zeros(st["weight_in"].shape, dtype=torch.float64, device="cuda")
    for i, length in enumerate(lengths):
        if weight is not None:
            weight[i, :, :length] = st["weight_in"][i, :, :length].double()
        for g in range(hkv):
            heads = slice(g * grp, (g + 1) * grp)
            for q0 in range(0, n, 1024):
                q1 = min(n, q0 + 1024)
                first, last = length - n + q0, length - n + q1 - 1   # positions of these queries
                low = 0 if c["window"] < 0 else max(0, first - c["window"] + 1)
                j = torch.cat([torch.arange(0, min(c["sinks"], low), device="cuda"),
                               torch.arange(low, last + 1, device="cuda")])
                kk, vv = cached("k", i, g, j), cached("v", i, g, j)
                q = st["q"][i, q0:q1, heads].double()
                z = torch.einsum("nhd,jd->nhj", q, kk) / math.sqrt(d)
                at = torch.arange(first, last + 1, device="cuda").view(-1, 1)
                hidden = j > at
                if c["window"] >= 0:
                    hidden |= (j <= at - c["window"]) & (j >= c["sinks"])
                z = z.masked_fill(hidden.unsqueeze(1), -INF)
                s = torch.logsumexp(z, -1)
                p = torch.exp(z - torch.where(s == -INF, torch.zeros_like(s), s).unsqueeze(-1))
                out[i, q0:q1, heads] = torch.einsum("nhj,jd->nhd", p, vv)
                lse[i, q0:q1, heads] = s
                if weight is not None:
                    weight[i, g].index_add_(0, j, p.sum((0, 1)))
    got = {"out": out, "lse": lse}
    return dict(got, weight=weight) if weight is not None else got
