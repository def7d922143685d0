"""Paged key / value caches: block tables and slot maps from request lengths, the cache's writes, and attention of new tokens over
it.  Plain forms, definitions in 64 bits, and the cases at which they are measured.

A case's `kind`
  "plan"      pages handed out and taken back for the requests' lengths, the rows' positions and cache slots
  "write"     keys and values of new tokens into their slots
  "attn"      attention of every request's new tokens over its cached keys (their own among them)
Fields
  requests, mix, rows, ctx, lens_seed
              number of requests, and their lengths: up to `ctx` tokens in the cache; new ones by `mix`: "decode" one each, "verify" 1 to
              `rows` each, "chunk" `rows` each, "mixed" chunks that share `rows` for every eighth request and one for the others
  page        tokens of a page
  dtype, head_dim, nq, nkv, cut_map
              element type, columns, heads; the head map is that of a head-parallel cut through a group, not the even one
  layout      "heads": a page holds head after head; "tokens": token after token
  window, sinks      0: every key up to the row's own; otherwise the window and the first tokens that stay visible
  shards      a request's keys are spread over so many devices and this one holds the middle part; results are partial, in fp32
  k_scale     standard deviation of K
  pressure    "plan": too few pages for all
  pad         rows behind the last request's, as a captured batch has them
  x_dtype, fused     "write": element type of the new keys and values; they are slices of a fused q / k / v tensor
"""
import math
import random

import torch

own = False
DEV = "cuda:0"


def _plan_case(name, requests, mix, rows, ctx, page, lens_seed, pressure=False, pad=0):
    c = dict(kind="plan", requests=requests, mix=mix, rows=rows, ctx=ctx, page=page, lens_seed=lens_seed, pressure=pressure, pad=pad)
    return dict(name=name, **c) if name else c


def _write_case(name, dtype, x_dtype, d, nq, nkv, rows, page, layout, fused, pad=0):
    c = dict(kind="write", dtype=dtype, x_dtype=x_dtype, head_dim=d, nq=nq, nkv=nkv, rows=rows, page=page, layout=layout, fused=fused, pad=pad)
    return dict(name=name, **c) if name else c


def _attn(name, dtype, d, nq, nkv, requests, mix, rows, ctx, page, layout, lens_seed, window=0, sinks=0, shards=1, k_scale=1.0, cut_map=False):
    c = dict(kind="attn", dtype=dtype, head_dim=d, nq=nq, nkv=nkv, requests=requests, mix=mix, rows=rows, ctx=ctx, page=page, layout=layout,
             lens_seed=lens_seed, window=window, sinks=sinks, shards=shards, k_scale=k_scale, cut_map=cut_map)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a decoding step of a serving batch, some of whose requests have ended
        _plan_case("plan_step", 64, "decode", 1, 12000, 16, 1),
        # a step that takes prompts in: 16K new tokens of 512 requests, fewer pages than they ask for
        _plan_case("plan_prompts", 512, "mixed", 16000, 4000, 16, 2, pressure=True, pad=384),
        # the step's keys and values, 8 kv heads
        _write_case("write_step", "bf16", "bf16", 128, 24, 8, 64, 16, "heads", True),
        # keys and values of a prompt of 16K tokens
        _write_case("write_prompt", "bf16", "bf16", 128, 24, 8, 16384, 64, "heads", True),
        # fp32 keys of 64 columns rounded into a bf16 cache that is laid out token by token; an odd number of rows, some of no slot
        _write_case("write_odd", "bf16", "f32", 64, 12, 4, 3001, 48, "tokens", False, pad=71),
        # one new token of one request, a 70B-like head group: latency
        _attn("attn_token", "bf16", 128, 8, 1, 1, "decode", 1, 2900, 16, "heads", 3),
        # a decoding batch of a 3B-like layer
        _attn("attn_batch", "bf16", 128, 24, 8, 48, "decode", 1, 12000, 16, "heads", 4),
        # two requests far into long contexts, one head group; this device's part of keys that lie on two
        _attn("attn_long", "bf16", 128, 8, 1, 2, "decode", 1, 900000, 64, "heads", 5, shards=2),
        # speculated tokens of requests with a window and sinks: several rows each, pages laid out token by token
        _attn("attn_verify", "bf16", 128, 32, 8, 24, "verify", 6, 60000, 32, "tokens", 6, window=4096, sinks=16),
        # numerics debugging in fp32: odd sizes, a head map cut through a group, pages of 48
        _attn("attn_fp32", "f32", 64, 7, 3, 5, "verify", 70, 3001, 48, "tokens", 7, cut_map=True),
        # chunks of prompts beside decoding requests, 64-column heads
        _attn("attn_mixed", "bf16", 64, 24, 8, 25, "mixed", 1400, 9000, 32, "heads", 8, k_scale=3.0),
        # a chunk of 2048 tokens of a long prompt
        _attn("attn_chunk", "bf16", 128, 24, 8, 1, "chunk", 2048, 32768, 64, "heads", 9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["plan", "plan", "write", "write", "attn", "attn", "attn", "attn", "attn"])
        page, seed = rng.choice([16, 16, 32, 48, 64, 128, 256]), rng.randint(1, 9999)
        d, layout = rng.choice([128, 128, 64]), rng.choice(["heads", "heads", "tokens"])
        nkv = rng.choice([1, 2, 3, 4, 8])
        nq = nkv * rng.choice([1, 2, 3, 4, 5, 8])
        if nq > 32:
            continue
        if kind == "plan":
            n, mix = _log_int(rng, 1, 1024), rng.choice(["decode", "verify", "mixed"])
            rows = dict(decode=1, verify=rng.randint(2, 8), mixed=_log_int(rng, 64, 16384))[mix]
            return _plan_case(None, n, mix, rows, _log_int(rng, 100, 12000), page, seed, rng.random() < 0.3, rng.choice([0, 0, 1, 100]))
        if kind == "write":
            rows = _log_int(rng, 1, 16384)
            dtype = rng.choice(["bf16", "bf16", "f32"])
            return _write_case(None, dtype, rng.choice(["f32", dtype]), d, nq, nkv, rows if dtype == "bf16" else min(rows, 8192), page, layout,
                               rng.random() < 0.6, rng.choice([0, 0, 1, 50]))
        mix = rng.choice(["decode", "decode", "verify", "mixed", "chunk"])
        n = 1 if mix == "chunk" and rng.random() < 0.5 else _log_int(rng, 1, 64)
        rows = dict(decode=1, verify=_log_int(rng, 2, 64), mixed=_log_int(rng, 16, 4096), chunk=_log_int(rng, 16, 4096))[mix]
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        cut = nkv > 1 and nq > nkv and rng.random() < 0.2
        window = _log_int(rng, 16, 8192) if rng.random() < 0.3 else 0
        c = _attn(None, dtype, d, nq - 1 if cut else nq, nkv, n, mix, rows, _log_int(rng, 8, 500000 if n < 4 else 60000), page, layout, seed,
                  window, rng.choice([0, 4, 64]) if window else 0, rng.choice([1, 1, 1, 1, 2, 3]), rng.choice([1.0, 1.0, 3.0]), cut)
        lens = _lens(c)
        cells = c["nq"] * sum((k + a) * a for k, a in lens)
        values = sum(k + a for k, a in lens) * nkv * d
        if cells > (1e8 if dtype == "f32" else 1.6e9) or values > (1.2e8 if dtype == "f32" else 2.4e8):
            continue
        return c


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _pages(tokens, page):
    return -(-tokens // page)


# ---- lengths ----

def _lens(c):
    """(tokens in the cache, new tokens) of every request."""
    rng = random.Random(c["lens_seed"])
    n, out = c["requests"], []
    chunks = _pages(n, 8)
    for r in range(n):
        cached = rng.randint(c["ctx"] // 2 if n < 4 else c["ctx"] // 16, c["ctx"])
        added = 1
        if c["mix"] == "verify":
            added = rng.randint(1, c["rows"])
        elif c["mix"] == "chunk":
            added = c["rows"]
        elif c["mix"] == "mixed" and r % 8 == 0:
            share = c["rows"] // chunks
            added = max(1, share - rng.randint(0, share // 4))
        out.append((cached, added))
    return out


def _plan_lens(c):
    """(tokens that stay, new tokens, pages held before): some requests have ended or lost speculated tokens."""
    rng = random.Random(c["lens_seed"] + 17)
    out = []
    for r, (cached, added) in enumerate(_lens(c)):
        x = rng.random() if r else 1.0
        held = _pages(cached, c["page"])
        if x < 0.04:
            cached = added = 0
        elif x < 0.08:
            held += rng.randint(1, 4)
        elif x < 0.12:
            added = 0
        out.append((cached, added, held))
    return out


def _spans(c):
    """Of every request of an "attn" case: (keys in this device's cache, position of the first of them, new tokens, position of the first row)."""
    out = []
    for cached, added in _lens(c):
        if c["shards"] == 1:
            out.append((cached + added, 0, added, cached))
        else:
            part = _pages(cached, c["shards"])
            out.append((min(part, cached), part * ((c["shards"] - 1) // 2), added, cached))
    return out


def _kv_of_q(c):
    if not c["cut_map"]:
        return [h // (c["nq"] // c["nkv"]) for h in range(c["nq"])]
    g = (c["nq"] + c["nkv"]) // c["nkv"]      # group size before the cut; the first head of the first group is elsewhere
    return [min((h + 1) // g, c["nkv"] - 1) for h in range(c["nq"])]


# ---- inputs ----

def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 29)

    def normal(shape, dtype, std=1.0):
        return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEV)

    def shuffled(n):
        return torch.randperm(n, generator=gen, device=DEV).to(torch.int32)

    st = dict(case=c)
    if c["kind"] == "plan":
        lens = _plan_lens(c)
        held, asked = [h for _, _, h in lens], sum(max(0, _pages(k + a, c["page"]) - h) for k, a, h in lens)
        columns = max(max(h, _pages(k + a, c["page"])) for k, a, h in lens) + 3
        spare = asked // 2 if c["pressure"] else asked + 100
        ids = shuffled(sum(held) + spare)
        table = torch.zeros((len(lens), columns), dtype=torch.int32, device=DEV)
        at = 0
        for r, h in enumerate(held):
            table[r, :h] = ids[at:at + h]
            at += h
        free = torch.zeros(ids.numel(), dtype=torch.int32, device=DEV)
        free[:spare] = ids[at:]
        rows = sum(a for _, a, _ in lens) + c["pad"]
        return st | dict(cached=ints([k for k, _, _ in lens]), added=ints([a for _, a, _ in lens]), held=ints(held), table=table, free=free,
                         n_free=ints([spare]), n_rows=rows)
    d, nkv, page = c["head_dim"], c["nkv"], c["page"]

    def cache(n_pages, std):       # [pages][heads][page][columns], whatever lies beside what in memory
        if c["layout"] == "heads":
            return normal((n_pages, nkv, page, d), _type(c["dtype"]), std)
        return normal((n_pages, page, nkv, d), _type(c["dtype"]), std).transpose(1, 2)

    if c["kind"] == "write":
        rows, xt = c["rows"], _type(c["x_dtype"])
        n_pages = _pages(rows, page) + 5
        pages = shuffled(n_pages)
        r = torch.arange(rows, device=DEV)
        slot = torch.full((rows + c["pad"],), -1, dtype=torch.int32, device=DEV)
        slot[:rows] = (pages[r // page].long() * page + r % page).to(torch.int32)
        if c["fused"]:
            x = normal((rows + c["pad"], c["nq"] + 2 * nkv, d), xt)
            k, v = x[:, c["nq"]:c["nq"] + nkv], x[:, c["nq"] + nkv:]
        else:
            k, v = normal((rows + c["pad"], nkv, d), xt), normal((rows + c["pad"], nkv, d), xt)
        return st | dict(slot=slot, k=k, v=v, k_cache=cache(n_pages, 1.0), v_cache=cache(n_pages, 1.0))
    spans = _spans(c)
    counts = [_pages(n, page) for n, _, _, _ in spans]
    pages = shuffled(sum(counts) + 5)
    table = torch.zeros((len(spans), max(counts) + 3), dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(counts):
        table[r, :n] = pages[at:at + n]
        at += n
    starts = [0]
    for _, _, n, _ in spans:
        starts.append(starts[-1] + n)
    st |= dict(q=normal((starts[-1], c["nq"], d), _type(c["dtype"])), k_cache=cache(sum(counts) + 5, c["k_scale"]), v_cache=cache(sum(counts) + 5, 1.0),
               table=table, row_start=ints(starts), kv_len=ints([n for n, _, _, _ in spans]))
    if c["shards"] > 1:
        st |= dict(q_start=ints([p for _, _, _, p in spans]), kv_start=ints([p for _, p, _, _ in spans]))
    return st


# ---- plain forms ----

def _plain_plan(st):
    c, page = st["case"], st["case"]["page"]
    table, free, n_rows = st["table"], st["free"], st["n_rows"]
    cached, added, held = st["cached"].long(), st["added"].long(), st["held"].long()
    end = torch.cumsum(added, 0)
    want = (cached + added + page - 1) // page
    keep = torch.minimum(held, want)
    # back: request by request, page by page, onto the free list
    back = held - keep
    n, request = int(back.sum()), torch.arange(len(back), device=DEV)
    owner = torch.repeat_interleave(request, back, output_size=n)
    nth = torch.arange(n, device=DEV) - (torch.cumsum(back, 0) - back)[owner]
    count = st["n_free"].long()
    free[count + torch.arange(n, device=DEV)] = table[owner, keep[owner] + nth]
    count = count + n
    # out: from the end of the list, to the requests that can have all that they need
    need = want - keep
    got = torch.where((torch.cumsum(need, 0) <= count) & (want <= table.shape[1]) & (end <= n_rows), need, torch.zeros_like(need))
    granted = got == need
    n = int(got.sum())
    owner = torch.repeat_interleave(request, got, output_size=n)
    nth = torch.arange(n, device=DEV) - (torch.cumsum(got, 0) - got)[owner]
    table[owner, keep[owner] + nth] = free[count - 1 - torch.arange(n, device=DEV)]
    st["n_free"].copy_((count - n).to(torch.int32))
    st["held"].copy_((keep + got).to(torch.int32))
    kv_len = torch.where(granted, cached + added, torch.minimum(cached, keep * page))
    # rows
    row = torch.arange(n_rows, device=DEV)
    owner = torch.searchsorted(end, row, right=True)
    real = owner < len(end)
    owner = owner.clamp(max=len(end) - 1)
    pos = cached[owner] + row - (end - added)[owner]
    slot = table[owner, (pos // page).clamp(max=table.shape[1] - 1)].long() * page + pos % page
    slot = torch.where(real & (pos < kv_len[owner]), slot, torch.full_like(slot, -1))
    pos = torch.where(real, pos, torch.zeros_like(pos))
    row_start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), end])
    ints = [x.to(torch.int32) for x in (row_start, kv_len, pos, slot)]
    return (table, st["held"], free, st["n_free"], *ints)


def _plain_write(st):
    page, slot = st["case"]["page"], st["slot"].long()
    rows = torch.nonzero(slot >= 0).flatten()
    at = slot[rows]
    for new, cache in ((st["k"], st["k_cache"]), (st["v"], st["v_cache"])):
        cache[at // page, :, at % page] = new[rows].to(cache.dtype)
    return st["k_cache"], st["v_cache"]


def _request(st, r):
    """A request's rows and its keys and values, one of each for every q head, in fp32; the mask."""
    c = st["case"]
    n, kv_start, added, q_start = _spans(c)[r]
    first = sum(a for _, _, a, _ in _spans(c)[:r])
    pages = st["table"][r, :_pages(n, c["page"])].long()
    k, v = (st[x][pages].transpose(0, 1).flatten(1, 2)[:, :n].float()[_kv_of_q(c)] for x in ("k_cache", "v_cache"))
    q = st["q"][first:first + added].float().transpose(0, 1).contiguous()
    p, j = torch.arange(added, device=DEV)[:, None] + q_start, torch.arange(n, device=DEV)[None, :] + kv_start
    seen = j <= p
    if c["window"]:
        seen &= (p - j < c["window"]) | (j < c["sinks"])
    return slice(first, first + added), q, k, v, seen


def _plain_attn(st):
    c = st["case"]
    o = torch.zeros(st["q"].shape, device=DEV)
    lse = torch.empty((c["nq"], o.shape[0]), device=DEV)
    for r in range(c["requests"]):
        rows, q, k, v, seen = _request(st, r)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(c["head_dim"]))
        s = s.masked_fill_(~seen, -math.inf)
        m = s.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        p = s.sub_(m).exp_()
        total = p.sum(-1, keepdim=True)
        o[rows] = (torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)).transpose(0, 1)
        lse[:, rows] = (m + total.log()).squeeze(-1)
    return o.to(_out_type(c)), lse


def _out_type(c):
    return _type(c["dtype"]) if c["shards"] == 1 else torch.float32


# ---- the framework's operators ----

def _plan(st):
    """What a program keeps from call to call: descriptors, output buffers, workspace."""
    from paper_2605_07569_amd import hexi
    c = st["case"]
    p = dict(hexi=hexi)

    def ints(n):
        return torch.empty((n,), dtype=torch.int32, device=DEV)

    if c["kind"] == "plan":
        return p | dict(row_start=ints(c["requests"] + 1), kv_len=ints(c["requests"]), pos=ints(st["n_rows"]), slot=ints(st["n_rows"]))
    p["cache"] = hexi.make_paged_cache(st["k_cache"])
    if c["kind"] == "write":
        return p
    rows, most = st["q"].shape[0], max(a for _, _, a, _ in _spans(c))
    p |= dict(desc=hexi.paged_desc_for(st["q"], st["k_cache"], 1.0 / math.sqrt(c["head_dim"]), _kv_of_q(c) if c["cut_map"] else None),
              window=hexi.make_window(c["window"], c["sinks"]) if c["window"] else None, max_rows=most,
              o=torch.empty(st["q"].shape, dtype=_out_type(c), device=DEV), lse=torch.empty((c["nq"], rows), device=DEV))
    n = hexi.hexi_paged_attn_workspace_bytes(p["desc"], p["cache"], c["requests"], st["table"].shape[1], rows, most)
    return p | dict(workspace=torch.empty((n,), dtype=torch.uint8, device=DEV) if n else None)


def run(state):
    st = state
    c = st["case"]
    if not own:
        return dict(plan=_plain_plan, write=_plain_write, attn=_plain_attn)[c["kind"]](st)
    p = st.get("plan")
    if p is None:
        p = st["plan"] = _plan(st)
    hexi = p["hexi"]
    if c["kind"] == "plan":
        hexi.hexi_paged_plan(c["page"], st["cached"], st["added"], st["table"], st["held"], st["free"], st["n_free"], p["row_start"], p["kv_len"],
                             p["pos"], p["slot"])
        return st["table"], st["held"], st["free"], st["n_free"], p["row_start"], p["kv_len"], p["pos"], p["slot"]
    if c["kind"] == "write":
        hexi.hexi_paged_write(p["cache"], st["slot"], st["k"], st["v"], st["k_cache"], st["v_cache"])
        return st["k_cache"], st["v_cache"]
    hexi.hexi_paged_attn(p["desc"], p["cache"], st["table"], st["row_start"], st["kv_len"], st["q"], st["k_cache"], st["v_cache"], p["o"], p["lse"],
                         max_rows=p["max_rows"], window=p["window"], q_start=st.get("q_start"), kv_start=st.get("kv_start"), workspace=p["workspace"])
    return p["o"], p["lse"]


# ---- floors and definitions ----

def _visible(c, span):
    """Visible (row, key) pairs of a request, and keys that some row sees."""
    n, kv_start, added, q_start = span
    p = torch.arange(q_start, q_start + added, dtype=torch.int64) - kv_start      # keys 0 .. n - 1 of the cache
    hi = torch.clamp(p + 1, min=0, max=n)
    if not c["window"]:
        return int(hi.sum()), int(hi.max())
    lo = torch.minimum(torch.clamp(p - c["window"] + 1, min=0), hi)
    sink = torch.clamp(torch.minimum(torch.tensor(c["sinks"] - kv_start), lo), min=0)
    return int((hi - lo + sink).sum()), int(hi.max() - lo.min() + torch.minimum(sink.max(), lo.min()))


def work(case):
    c = case
    if c["kind"] == "plan":
        rows, n = sum(a for _, a, _ in _plan_lens(c)), c["requests"]
        # lengths and pages held in, pages held, row starts and key lengths out; of a row its page, its position and its slot
        return dict(bytes=4 * (6 * n + 1) + 4 * _pages(rows, c["page"]) + 8 * (rows + c["pad"]), flops=4 * n + 4 * rows)
    e, d, nkv = (2 if c["dtype"] == "bf16" else 4), c["head_dim"], c["nkv"]
    if c["kind"] == "write":
        return dict(bytes=2 * c["rows"] * nkv * d * (e + (2 if c["x_dtype"] == "bf16" else 4)) + 4 * (c["rows"] + c["pad"]), flops=0)
    spans = _spans(c)
    rows, seen = sum(s[2] for s in spans), [_visible(c, s) for s in spans]
    used = len(set(_kv_of_q(c)))
    out = 2 if _out_type(c) == torch.bfloat16 else 4
    return dict(bytes=rows * c["nq"] * (d * (e + out) + 4) + sum(k for _, k in seen) * 2 * used * d * e + 4 * sum(_pages(k, c["page"]) for _, k in seen),
                flops=4 * d * c["nq"] * sum(pairs for pairs, _ in seen))


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "plan":
        return _exact_plan(st)
    if c["kind"] == "write":
        out = []
        for new, cache in ((st["k"], st["k_cache"]), (st["v"], st["v_cache"])):
            y = cache.double()
            flat = y.transpose(1, 2).reshape(-1, c["nkv"], c["head_dim"])      # by slot
            keep = st["slot"] >= 0
            flat = flat.index_copy(0, st["slot"][keep].long(), new[keep].double())
            out.append(flat.view(-1, c["page"], c["nkv"], c["head_dim"]).transpose(1, 2))
        return tuple(out)
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty((c["nq"], o.shape[0]), dtype=torch.float64, device=DEV)
    kv, first = _kv_of_q(c), 0
    for r, (n, kv_start, added, q_start) in enumerate(_spans(c)):
        j = torch.arange(n, device=DEV)
        page, within = st["table"][r][j // c["page"]].long(), j % c["page"]
        where = j.double() + kv_start
        for h in range(c["nq"]):
            k, v = st["k_cache"][page, kv[h], within].double(), st["v_cache"][page, kv[h], within].double()
            for i in range(0, added, 2048):
                rows = slice(first + i, first + min(i + 2048, added))
                dist = torch.arange(i, min(i + 2048, added), device=DEV).double()[:, None] + q_start - where[None, :]
                seen = dist >= 0
                if c["window"]:
                    seen = torch.logical_and(seen, torch.logical_or(dist <= c["window"] - 1, (where <= c["sinks"] - 1)[None, :].expand_as(dist)))
                s = torch.where(seen, torch.mm(st["q"][rows, h].double(), k.t()) / math.sqrt(c["head_dim"]), torch.full_like(dist, -math.inf))
                logz = torch.logsumexp(s, 1)
                lse[h, rows] = logz
                w = torch.where(seen, torch.exp(s - torch.where(torch.isinf(logz), torch.zeros_like(logz), logz)[:, None]), torch.zeros_like(s))
                o[rows, h] = torch.mm(w, v)
        first += added
    return o, lse


def _exact_plan(st):
    """The rules one request, page and row at a time, on the host."""
    page, n_rows = st["case"]["page"], st["n_rows"]
    cached, added, held, free = (st[x].tolist() for x in ("cached", "added", "held", "free"))
    table, top, total = st["table"].cpu(), int(st["n_free"][0]), 0
    row_start, kv_len, pos, slot = [0], [], [], []
    for r in range(len(held)):
        while held[r] * page >= cached[r] + added[r] + page:      # a page more than the request's tokens fill
            top, held[r] = top + 1, held[r] - 1
    # (what a request gives back goes onto the list in the order of its pages)
    at = int(st["n_free"][0])
    for r, before in enumerate(st["held"].tolist()):
        for i in range(held[r], before):
            free[at] = int(table[r, i])
            at += 1
    budget, asked = top, 0
    for r in range(len(held)):
        need = 0
        while (held[r] + need) * page < cached[r] + added[r]:
            need += 1
        asked += need
        total += added[r]
        fits = asked <= budget and held[r] + need <= table.shape[1] and total <= n_rows
        if fits:
            for _ in range(need):
                top -= 1
                table[r, held[r]] = free[top]
                held[r] += 1
        kv_len.append(cached[r] + added[r] if fits else min(cached[r], held[r] * page))
        row_start.append(total)
        for i in range(cached[r], cached[r] + added[r]):
            pos.append(i)
            slot.append(int(table[r, i // page]) * page + i % page if fits else -1)
    pos += [0] * (n_rows - len(pos))
    slot += [-1] * (n_rows - len(slot))
    return tuple(torch.tensor(x, device=DEV).reshape(s) for x, s in
                 ((table.tolist(), table.shape), (held, (-1,)), (free, (-1,)), ([top], (1,)), (row_start, (-1,)), (kv_len, (-1,)), (pos, (-1,)), (slot, (-1,))))
