"""The operators of the 8-bit cache, as cases that can be timed: what a serving program's forward pass asks of one layer's cache.

A case is one of these kinds of pass:

  append   new keys and values go into pages of e4m3 with a power-of-two scale per (page, KV head, keys | values), normalised per
           head and rotated on the way, the queries with them
  attend   attention of a packed batch's rows over all tokens their sequences hold, each row up to its own position
  sparse   per row and KV head a list of pages chosen by the bounds of their keys, then attention over those pages alone

Sequences have ragged lengths and scattered pages.  Keys, values and queries are those of the repository's workloads: per KV head a
unit direction u, heavy keys 4u + 0.1 N(0, I) with a probability of the sequence's own, other keys and all values N(0, I), queries
2u + N(0, I).  With `own` the framework's kernels run, without it the same definitions in elementary torch operations.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
E_MIN, E_MAX = -117, 119       # exponents a page's scale may take
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(kind, name=None, **kw):
    """hq, hkv, d: heads and their size; page: tokens per page; seqs sequences of lo to hi tokens, the last rows_lo to rows_hi of which
    (all of them where whole) are the batch's rows; first, recent, keep: pages always taken, pages taken in all."""
    c = dict(kind=kind, hq=32, hkv=8, d=128, page=16, dtype="bf16", out="bf16", seqs=1, lo=1, hi=1, rows_lo=1, rows_hi=1, whole=False, shape=1)
    if kind == "append":
        c.update(theta=1e6, norm=True, shift=0)
    if kind == "sparse":
        c.update(keep=64, first=1, recent=2)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # A handful of chats, a token each: launches and latency are everything.
        _case("append", "append_tokens", seqs=8, lo=20, hi=500),
        # Throughput serving, a token each; positions ahead of the slots, as where a cache has dropped tokens.
        _case("append", "append_tokens_batch", seqs=256, lo=60, hi=3000, page=64, shift=5000, shape=2),
        # New requests: whole prompts of odd lengths, normalised and rotated.
        _case("append", "append_prompts", seqs=7, lo=3, hi=4099, whole=True, shape=3),
        # Chunks of long prompts that begin inside a page, half precision, small heads in groups of eight, no normalisation.
        _case("append", "append_chunks_f16", seqs=5, hq=64, d=64, page=32, dtype="f16", norm=False, theta=1e4, lo=900, hi=20000,
              rows_lo=200, rows_hi=901, shape=4),
        # One chat of a few hundred tokens.
        _case("attend", "attend_one", lo=703, hi=703),
        # The repository's batch: 64 requests, a token each.
        _case("attend", "attend_batch", seqs=64, lo=60, hi=4000, shape=5),
        # A few very long generations in groups of eight, outputs in full precision.
        _case("attend", "attend_long", seqs=3, hq=64, page=64, lo=60001, hi=131071, out="f32", shape=6),
        # Drafted tokens: five rows a request, small heads, half precision.
        _case("attend", "attend_drafts", seqs=48, d=64, dtype="f16", out="f16", lo=200, hi=6000, rows_lo=5, rows_hi=5, shape=7),
        # Chunked prefill: hundreds of rows over what is held already.
        _case("attend", "attend_chunks", seqs=3, lo=1500, hi=9000, rows_lo=301, rows_hi=1101, shape=8),
        # One long chat on a budget of 64 pages.
        _case("sparse", "sparse_one", lo=30011, hi=30011),
        # A batch of long chats on a budget of 128 pages.
        _case("sparse", "sparse_batch", seqs=48, lo=4000, hi=40000, keep=128, shape=9),
        # Large pages, groups of eight, two rows a request, half precision.
        _case("sparse", "sparse_page_64", seqs=16, hq=64, d=64, page=64, dtype="f16", out="f16", lo=3000, hi=30000, rows_lo=2, rows_hi=2, keep=33,
              shape=10),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hkv = rng.choice([1, 2, 4, 8])
    c = dict(hkv=hkv, hq=hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), d=rng.choice([64, 128]), page=rng.choice([16, 16, 32, 64, 128]),
             dtype=rng.choice(["bf16", "f16"]), shape=rng.randrange(1 << 20))
    kind = rng.choice(["append", "attend", "sparse"])
    c["out"] = rng.choice([c["dtype"], "f32"])
    if kind == "append":
        c.update(theta=rng.choice([0.0, 1e4, 1e6]), norm=rng.random() < 0.5, shift=rng.choice([0, 0, 131, 70000]))
        if rng.random() < 0.5:
            hi = _log(rng, 8, 8000)
            return _case(kind, seqs=min(_log(rng, 1, 256), 1 + 400000 // hi), lo=1, hi=hi, **c)
        hi = _log(rng, 8, 4100)
        return _case(kind, seqs=_log(rng, 1, 8), lo=1, hi=hi, whole=True, **c)
    if kind == "attend":
        if rng.random() < 0.6:
            hi = _log(rng, 2, 100000)
            return _case(kind, seqs=min(_log(rng, 1, 64), 1 + 250000 // hi), lo=max(1, hi // 50), hi=hi, **c)
        rows, hi = _log(rng, 2, 700), _log(rng, 16, 7000)
        return _case(kind, seqs=min(_log(rng, 1, 32), 1 + 900 // rows), lo=1, hi=max(rows, hi), rows_lo=1, rows_hi=rows, **c)
    hi = _log(rng, 64, 60000)
    keep = _log(rng, 3, 150)
    return _case(kind, seqs=min(_log(rng, 1, 48), 1 + 700000 // hi), lo=max(1, hi // 20), hi=hi, rows_hi=rng.choice([1, 1, 3]), keep=keep,
                 first=rng.choice([0, 1]), recent=rng.choice([1, 2]), **c)


# ------------------------------------------------------------------------------------------------ shapes and inputs
def _lens(c):
    """Tokens held and rows of the batch, per sequence."""
    r = random.Random(c["shape"])
    lens = [r.randint(c["lo"], c["hi"]) for _ in range(c["seqs"])]
    lens[0] = c["hi"]
    rows = [n if c["whole"] else min(n, r.randint(c["rows_lo"], c["rows_hi"])) for n in lens]
    return lens, rows


def _visible(c):
    """Tokens each row sees."""
    lens, rows = _lens(c)
    return [n - r + i + 1 for n, r in zip(lens, rows) for i in range(r)]


def work(c):
    lens, rows = _lens(c)
    hq, hkv, d, page, nrows = c["hq"], c["hkv"], c["d"], c["page"], sum(rows)
    table = 4 * sum(-(-n // page) for n in lens)
    if c["kind"] == "append":
        touched = sum((n - 1) // page - (n - r) // page + 1 for n, r in zip(lens, rows))
        inputs = nrows * (hq + 2 * hkv) * d * 2
        return {"bytes": inputs + nrows * (hq * d * 2 + hkv * 2 * d) + touched * hkv * (8 + 2 * d + 4), "flops": nrows * (hq + hkv) * d * 10}
    ends = nrows * hq * d * (2 + (4 if c["out"] == "f32" else 2))
    vis = _visible(c)
    if c["kind"] == "attend":
        return {"bytes": sum(lens) * hkv * 2 * d + sum(-(-n // page) for n in lens) * hkv * 8 + table + ends, "flops": 4 * hq * d * sum(vis)}
    kept = sum(min(-(-n // page), c["keep"]) for n in vis)
    scored = sum(-(-n // page) for n in lens)
    return {"bytes": scored * hkv * (2 * d + 4) + table + kept * hkv * (page * 2 * d + 8 + 4) + ends,
            "flops": 4 * hkv * d * sum(-(-n // page) for n in vis) + 4 * hq * d * kept * page}


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, for 64-bit amax; 448 = 0.875 * 2^9."""
    f, x = torch.frexp(amax)
    e = x - 9 + (f > 0.875).to(x.dtype)
    return torch.where(amax > 0, e.clamp(E_MIN, E_MAX), torch.full_like(e, E_MIN)).to(torch.int32)


def _codes(x):
    """64-bit values in a page's scale to e4m3: to 32 bits, then to the nearest code, at most 448 in magnitude; what is not finite becomes NaN."""
    y = x.to(torch.float32)
    return torch.where(torch.isfinite(y), y.clamp(-448.0, 448.0), torch.full_like(y, float("nan"))).to(torch.float8_e4m3fn)


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + 17)
    lens, rows = _lens(c)
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    dt = DTYPES[c["dtype"]]
    need = [-(-n // page) for n in lens]
    n_pages, width = sum(need) + 3, max(need)
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    owner = torch.empty(sum(need), dtype=torch.int64, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = perm[at:at + n]
        owner[at:at + n] = s
        at += n
    nrows = sum(rows)
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    u = torch.randn(hkv, d, generator=g, device=DEV)
    u = u / u.norm(dim=1, keepdim=True)
    heavy = 0.02 + 0.1 * torch.rand(len(lens), generator=g, device=DEV)

    def keys(who, n):
        x = torch.randn(n, hkv, d, generator=g, device=DEV)
        hot = torch.rand(n, hkv, 1, generator=g, device=DEV) < heavy[who].view(n, 1, 1)
        return torch.where(hot, 4 * u + 0.1 * x, x)

    # the cache as it is before the pass: every page filled (behind a sequence's end lies what an earlier owner left there)
    codes = torch.empty(n_pages, hkv, 2, page, d, dtype=torch.float8_e4m3fn, device=DEV)
    scales = torch.empty(n_pages, hkv, 2, dtype=torch.float32, device=DEV)
    bounds = torch.empty(n_pages, hkv, 2, d, dtype=torch.float8_e4m3fn, device=DEV)
    step = max(1, (1 << 25) // (page * hkv * d))
    order = perm.long()
    for a in range(0, n_pages, step):
        ids = order[a:a + step]
        n = len(ids)
        who = owner[a:a + n]
        who = torch.cat([who, who.new_zeros(n - len(who))]).repeat_interleave(page)
        kv = torch.stack([keys(who, n * page), torch.randn(n * page, hkv, d, generator=g, device=DEV)], 2).to(dt)
        kv = kv.view(n, page, hkv, 2, d).permute(0, 2, 3, 1, 4).contiguous().float()
        e = _exponent(kv.abs().amax((3, 4)).double())
        held = _codes(torch.ldexp(kv, -e[..., None, None]))
        codes.view(torch.uint8)[ids] = held.view(torch.uint8)
        scales[ids] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
        # bounds of the tokens a sequence holds: its last page may be part full (the rows behind its end count for nothing)
        bounds.view(torch.uint8)[ids] = torch.stack([held[:, :, 0].float().amin(2), held[:, :, 0].float().amax(2)], 2).to(torch.float8_e4m3fn).view(torch.uint8)
    s = dict(case=c, codes=codes, scales=scales, bounds=bounds, table=table,
             row_start=torch.tensor(start, dtype=torch.int32, device=DEV), seq_len=torch.tensor(lens, dtype=torch.int32, device=DEV),
             n_rows=nrows, max_rows=max(rows), max_len=max(lens))
    # bounds of pages that are part full: over the rows that a sequence holds once (append: before) the batch is in
    held_to = [n - r for n, r in zip(lens, rows)] if c["kind"] == "append" else lens
    part = [(i, n // page, n % page) for i, n in enumerate(held_to) if n % page]
    if part:
        ids = torch.stack([table[i, p] for i, p, _ in part]).long()
        keep = torch.tensor([k for _, _, k in part], device=DEV).view(-1, 1, 1, 1)
        x = codes.view(torch.uint8)[ids][:, :, 0].view(torch.float8_e4m3fn).float()
        slot = torch.arange(page, device=DEV).view(1, 1, -1, 1)
        lo = torch.where(slot < keep, x, torch.full_like(x, 1e9)).amin(2)
        hi = torch.where(slot < keep, x, torch.full_like(x, -1e9)).amax(2)
        bounds.view(torch.uint8)[ids] = torch.stack([lo, hi], 2).to(torch.float8_e4m3fn).view(torch.uint8)
    who = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(rows, device=DEV))
    q = 2 * u.repeat_interleave(hq // hkv, 0) + torch.randn(nrows, hq, d, generator=g, device=DEV)
    if c["kind"] != "append":
        s["q"] = q.to(dt)
        return s
    # queries, keys and values are slices of one projection's output, as a model has them
    k = keys(who, nrows)
    v = torch.randn(nrows, hkv, d, generator=g, device=DEV)
    qkv = torch.cat([q.reshape(nrows, -1), k.reshape(nrows, -1), v.reshape(nrows, -1)], 1).to(dt)
    s["qkv"] = qkv
    s["q"], s["k"], s["v"] = qkv[:, :hq * d].view(nrows, hq, d), qkv[:, hq * d:(hq + hkv) * d].view(nrows, hkv, d), qkv[:, (hq + hkv) * d:].view(nrows, hkv, d)
    slot = torch.cat([torch.arange(n - r, n) for n, r in zip(lens, rows)])
    s["positions"] = (slot + c["shift"]).to(torch.int32).to(DEV)
    if c["norm"]:
        s["q_weight"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV)
        s["k_weight"] = 1 + 0.2 * torch.randn(d, generator=g, device=DEV)
    # the pages the batch writes: sequence, place in its table, rows held before, rows held after
    touched = [(i, p, min(page, max(0, n - r - p * page)), min(page, n - p * page))
               for i, (n, r) in enumerate(zip(lens, rows)) for p in range((n - r) // page, (n - 1) // page + 1)]
    s["touched"] = torch.tensor(touched, dtype=torch.int64, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ a pass
def _handle(s):
    """The cache and the batch as a program keeps them: descriptions of tensors that it owns."""
    if "cache" not in s:
        from paper_2609_03494_b200 import binding as B
        s["cache"] = B.QCache(s["codes"], s["scales"], s["bounds"])
        s["batch"] = B.QBatch(s["row_start"], s["seq_len"], s["table"], s["n_rows"], s["max_rows"], s["max_len"])
    return s["cache"], s["batch"]


def run(s):
    c = s["case"]
    if own:
        cache, batch = _handle(s)
        if c["kind"] == "append":
            q_out = cache.append(batch, s["k"], s["v"], q=s["q"], positions=s["positions"], rope_theta=c["theta"], q_weight=s.get("q_weight"),
                                 k_weight=s.get("k_weight"), eps=1e-6)
            return {"codes": s["codes"], "scales": s["scales"], "bounds": s["bounds"], "q": q_out}
        out = DTYPES[c["out"]]
        if c["kind"] == "attend":
            return {"out": cache.attention(batch, s["q"], out_dtype=out)}
        pages = cache.select(batch, s["q"], c["keep"], c["first"], c["recent"])
        return {"pages": pages, "out": cache.attention(batch, s["q"], out_dtype=out, pages=pages)}
    if c["kind"] == "append":
        return _plain_append(s)
    if c["kind"] == "attend":
        return {"out": _plain_attend(s)}
    pages = _plain_select(s)
    return {"pages": pages, "out": _plain_sparse(s, pages)}


def _rows(s):
    """Per row of the batch: its sequence and its position."""
    row = torch.arange(s["n_rows"], device=DEV)
    who = torch.searchsorted(s["row_start"][1:].long(), row, right=True)
    n_rows = (s["row_start"][1:] - s["row_start"][:-1]).long()
    return who, s["seq_len"].long()[who] - n_rows[who] + row - s["row_start"].long()[who]


def _norm_rotate(x, weight, positions, theta):
    x = x.double()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.double()
    if theta:
        h = x.shape[-1] // 2
        freq = theta ** (-torch.arange(h, device=DEV, dtype=torch.float64) / h)
        a = positions.double()[:, None, None] * freq
        cos, sin = torch.cos(a), torch.sin(a)
        x = torch.cat([x[..., :h] * cos - x[..., h:] * sin, x[..., h:] * cos + x[..., :h] * sin], -1)
    return x


def _plain_append(s):
    c, codes, scales, bounds = s["case"], s["codes"], s["scales"], s["bounds"]
    page = c["page"]
    k = _norm_rotate(s["k"], s.get("k_weight"), s["positions"], c["theta"])
    q = _norm_rotate(s["q"], s.get("q_weight"), s["positions"], c["theta"]).float().to(s["q"].dtype)
    kv = torch.stack([k, s["v"].double()], 2)                                       # [rows][hkv][2][d]
    who, slot = _rows(s)
    ids = s["table"][who, slot // page].long()
    amax = torch.where(torch.isfinite(kv), kv.abs(), torch.zeros_like(kv)).amax(-1)
    top = torch.zeros(codes.shape[:3], dtype=torch.float64, device=DEV).scatter_reduce_(0, ids[:, None, None].expand_as(amax), amax, "amax")
    seq, place, before, after = s["touched"].unbind(1)
    tid = s["table"][seq, place].long()
    e_new, e_old = _exponent(top[tid]), torch.frexp(scales[tid])[1] - 1
    e = torch.where((before > 0)[:, None, None], torch.maximum(e_new, e_old), e_new)
    raw = codes.view(torch.uint8)
    old = raw[tid].view(torch.float8_e4m3fn).float()
    was = (torch.arange(page, device=DEV) < before[:, None])[:, None, None, :, None]
    kept = torch.where(was, _codes(torch.ldexp(old, (e_old - e)[..., None, None])).float(), old)
    raw[tid] = torch.where(was, kept.to(torch.float8_e4m3fn).view(torch.uint8), raw[tid])
    scales[tid] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
    mine = torch.ldexp(kv, (1 - torch.frexp(scales[ids])[1]).double()[..., None].to(torch.int32))
    raw[ids, :, :, slot % page] = _codes(mine).view(torch.uint8)
    held = raw[tid][:, :, 0].view(torch.float8_e4m3fn).float()
    counts = (torch.arange(page, device=DEV) < after[:, None])[:, None, :, None]
    held = torch.where(torch.isnan(held), torch.zeros_like(held), held)
    lo = torch.where(counts, held, torch.full_like(held, float("inf"))).amin(2)
    hi = torch.where(counts, held, torch.full_like(held, float("-inf"))).amax(2)
    both = torch.stack([lo, hi], 2)
    bounds.view(torch.uint8)[tid] = both.to(torch.float8_e4m3fn).view(torch.uint8)
    return {"codes": codes, "scales": scales, "bounds": bounds, "q": q}


def _padded_queries(s):
    """[seqs][max_rows][hkv][group][d] in 32 bits, and each row's place in it."""
    c = s["case"]
    who, pos = _rows(s)
    at = torch.arange(s["n_rows"], device=DEV) - s["row_start"].long()[who]
    q = torch.zeros(c["seqs"], s["max_rows"], c["hq"], c["d"], device=DEV)
    q[who, at] = s["q"].float()
    vis = torch.zeros(c["seqs"], s["max_rows"], dtype=torch.int64, device=DEV)
    vis[who, at] = pos + 1
    return q.view(c["seqs"], s["max_rows"], c["hkv"], c["hq"] // c["hkv"], c["d"]), vis, who, at


def _weights(x, seen):
    """exp(x - max) over what is seen and its sum; where nothing is seen, zeros over one."""
    x = torch.where(seen, x, torch.full_like(x, float("-inf")))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isfinite(m), m, torch.zeros_like(m)))
    l = p.sum(-1, keepdim=True)
    return p, torch.where(l > 0, l, torch.ones_like(l))


def _plain_attend(s):
    c = s["case"]
    q, vis, who, at = _padded_queries(s)
    n = s["table"].shape[1] * c["page"]
    ids = s["table"].clamp_min(0).long()
    kv = s["codes"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float() * s["scales"][ids][..., None, None]   # [B][pages][hkv][2][page][d]
    kv = kv.permute(3, 0, 2, 1, 4, 5).reshape(2, c["seqs"], c["hkv"], n, c["d"])
    held = (torch.arange(n, device=DEV) < s["seq_len"][:, None])[:, None, :, None]
    k, v = kv[0], torch.where(held, kv[1], torch.zeros((), device=DEV))
    qq = q.permute(0, 2, 1, 3, 4).reshape(c["seqs"], c["hkv"], -1, c["d"])                   # rows x group
    x = torch.matmul(qq, k.transpose(2, 3)) / math.sqrt(c["d"])
    seen = (torch.arange(n, device=DEV) < vis[:, :, None]).repeat_interleave(c["hq"] // c["hkv"], 1)[:, None]
    p, l = _weights(x, seen)
    o = torch.matmul(p, v) / l
    o = o.view(c["seqs"], c["hkv"], s["max_rows"], -1, c["d"]).permute(0, 2, 1, 3, 4).reshape(c["seqs"], s["max_rows"], c["hq"], c["d"])
    return o[who, at].to(DTYPES[c["out"]])


def _plain_select(s):
    c = s["case"]
    hkv, grp, d, keep = c["hkv"], c["hq"] // c["hkv"], c["d"], c["keep"]
    who, pos = _rows(s)
    q = s["q"].double().view(-1, hkv, grp, d)
    plus, minus = q.clamp_min(0).sum(2), q.clamp_max(0).sum(2)
    ids = s["table"].clamp_min(0).long()
    b = s["bounds"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).float().double() * s["scales"][ids][..., 0].double()[..., None, None]
    at = torch.arange(s["n_rows"], device=DEV) - s["row_start"].long()[who]
    pad = torch.zeros(2, c["seqs"], s["max_rows"], hkv, d, dtype=torch.float64, device=DEV)
    pad[0, who, at], pad[1, who, at] = plus, minus
    score = (torch.einsum("srhd,sphd->srhp", pad[0], b[:, :, :, 1]) + torch.einsum("srhd,sphd->srhp", pad[1], b[:, :, :, 0]))[who, at]
    n = (pos + c["page"]) // c["page"]                                                       # pages a row sees
    j = torch.arange(ids.shape[1], device=DEV)
    score = torch.where((j < c["first"]) | (j >= n[:, None] - c["recent"]), float("inf"), 0.0)[:, None] + score
    score = torch.where((j < n[:, None])[:, None], score, float("-inf"))
    order = torch.sort(score, dim=-1, descending=True, stable=True)
    got = torch.where(order.values[..., :keep] > float("-inf"), order.indices[..., :keep], torch.full_like(order.indices[..., :keep], 1 << 30))
    got = torch.sort(got, -1).values
    got = torch.where(got < (1 << 30), got, torch.full_like(got, -1)).to(torch.int32)
    return torch.nn.functional.pad(got, (0, keep - got.shape[-1]), value=-1)


def _plain_sparse(s, pages):
    c = s["case"]
    who, pos = _rows(s)
    hkv, grp, d, page = c["hkv"], c["hq"] // c["hkv"], c["d"], c["page"]
    ok = pages >= 0
    ids = s["table"][who[:, None, None], pages.clamp_min(0).long()].clamp_min(0).long()      # [rows][hkv][keep]
    head = torch.arange(hkv, device=DEV)[:, None]
    kv = s["codes"].view(torch.uint8)[ids, head].view(torch.float8_e4m3fn).float() * s["scales"][ids, head][..., None, None]
    slot = pages[..., None] * page + torch.arange(page, device=DEV)
    seen = (ok[..., None] & (slot <= pos[:, None, None, None])).reshape(*pages.shape[:2], 1, -1)
    k, v = kv[:, :, :, 0].reshape(*pages.shape[:2], -1, d), kv[:, :, :, 1].reshape(*pages.shape[:2], -1, d)
    v = torch.where(seen.transpose(2, 3), v, torch.zeros((), device=DEV))
    p, l = _weights(torch.matmul(s["q"].float().view(-1, hkv, grp, d), k.transpose(2, 3)) / math.sqrt(d), seen)
    return (torch.matmul(p, v) / l).reshape(-1, c["hq"], d).to(DTYPES[c["out"]])


# ------------------------------------------------------------------------------------------------ in 64 bits, from the definitions
def exact(c, seed):
    """Sequence by sequence.  Codes, bounds and 16-bit results are given unrounded; old rows of a page whose scale grows are the values they held."""
    s = prepare(c, seed)
    lens, rows = _lens(c)
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    grp, start = hq // hkv, 0
    two = lambda e: 2.0 ** e.double()  # noqa: E731
    values = lambda t, ids: t.view(torch.uint8)[ids].view(torch.float8_e4m3fn).double()  # noqa: E731
    if c["kind"] == "append":
        codes, scales, bounds = s["codes"].double(), s["scales"].double(), s["bounds"].double()
        q_out = torch.empty(sum(rows), hq, d, dtype=torch.float64, device=DEV)
        inv = torch.tensor([c["theta"] ** (-2.0 * i / d) if c["theta"] else 0.0 for i in range(d // 2)], dtype=torch.float64, device=DEV)
        for i, (n, r) in enumerate(zip(lens, rows)):
            part = slice(start, start + r)
            start += r
            new = {}
            for what in ("q", "k"):
                x = s[what][part].double()
                if c["norm"]:
                    x = x / torch.sqrt(torch.sum(x ** 2, -1, keepdim=True) / d + 1e-6) * s[what + "_weight"].double()
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"][part].double()[:, None] * inv)[:, None]
                z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
                new[what] = torch.cat([z.real, z.imag], -1)
            q_out[part] = new["q"]
            p0, p1 = (n - r) // page, (n - 1) // page + 1
            held = s["table"][i, p0:p1].long()
            first = (n - r) - p0 * page                                             # tokens the first page holds already
            old, e_old = codes[held[0], :, :, :first].clone(), torch.round(torch.log2(scales[held[0]]))
            full = torch.zeros((p1 - p0) * page, hkv, 2, d, dtype=torch.float64, device=DEV)
            full[first:first + r, :, 0], full[first:first + r, :, 1] = new["k"], s["v"][part].double()
            full = full.view(p1 - p0, page, hkv, 2, d).permute(0, 2, 3, 1, 4)
            amax = full.abs().amax((3, 4))
            e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-60) / 448.0))
            e = torch.where(amax > 448.0 * two(e), e + 1, torch.where(amax <= 448.0 * two(e - 1), e - 1, e)).clamp(E_MIN, E_MAX)
            if first:
                e[0] = torch.maximum(e[0], e_old)
            got = full / two(e)[..., None, None]
            got[0, :, :, :first] = old * two(e_old - e[0])[..., None, None]
            count = torch.full((p1 - p0,), page)
            count[-1] = n - (p1 - 1) * page
            count = count.to(DEV).view(-1, 1, 1, 1)
            at = torch.arange(page, device=DEV).view(1, 1, -1, 1)
            lo = torch.where(at < count, got[:, :, 0], math.inf).amin(2)
            hi = torch.where(at < count, got[:, :, 0], -math.inf).amax(2)
            fresh = (at < count)[:, :, None]
            codes[held] = torch.where(fresh, got, codes[held])
            scales[held], bounds[held] = two(e), torch.stack([lo, hi], 2)
        return {"codes": codes, "scales": scales, "bounds": bounds, "q": q_out}
    out = torch.zeros(sum(rows), hq, d, dtype=torch.float64, device=DEV)
    listed_pages = torch.full((sum(rows), hkv, c.get("keep", 1)), -1, dtype=torch.int32, device=DEV)
    for i, (n, r) in enumerate(zip(lens, rows)):
        held = s["table"][i, :-(-n // page)].long()
        for h in range(hkv):
            kv = values(s["codes"], held)[:, h] * s["scales"][held][:, h].double()[..., None, None]
            k, v = kv[:, 0].reshape(-1, d)[:n], kv[:, 1].reshape(-1, d)[:n]
            q = s["q"][start:start + r, h * grp:(h + 1) * grp].double()
            see = torch.arange(n, device=DEV) <= torch.arange(n - r, n, device=DEV)[:, None]
            if c["kind"] == "sparse":
                b = values(s["bounds"], held)[:, h] * s["scales"][held][:, h, 0].double()[:, None, None]
                for x in range(r):
                    seen = -(-(n - r + x + 1) // page)
                    score = torch.maximum(q[x, :, None] * b[None, :seen, 0], q[x, :, None] * b[None, :seen, 1]).sum((0, 2))
                    must = list(range(min(c["first"], seen))) + list(range(max(c["first"], seen - c["recent"]), seen))
                    rest = [j for j in sorted(range(seen), key=lambda j, v=score.tolist(): (-v[j], j)) if j not in set(must)]
                    take = sorted((must + rest)[:c["keep"]]) if seen > c["keep"] else list(range(seen))
                    listed_pages[start + x, h, :len(take)] = torch.tensor(take, dtype=torch.int32, device=DEV)
                    chosen = torch.zeros(len(held), dtype=torch.bool, device=DEV)
                    chosen[take] = True
                    see[x] &= chosen.repeat_interleave(page)[:n]
            logit = torch.einsum("rgd,nd->rgn", q, k) * d ** -0.5
            w = torch.softmax(logit.masked_fill(~see[:, None], -math.inf), -1)
            out[start:start + r, h * grp:(h + 1) * grp] = torch.einsum("rgn,nd->rgd", w, v)
        start += r
    return {"pages": listed_pages, "out": out} if c["kind"] == "sparse" else {"out": out}
