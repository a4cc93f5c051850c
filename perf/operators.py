"""Performance cases of the serving operators: page maps, the paged K/V cache,
attention over it, and prefill attention with modified scores.

A case is one call that a serving program makes in a step (``map`` once a
step; ``write`` and ``paged`` once a layer) or in a prefill (``scored``, one
layer).  With ``own`` set, ``run`` makes the framework's call; without it, the
same result is computed from elementary torch operations in fp32.

Fields of a case (beside name and op)
  map     batch, cached and new lengths, page size, spare slots at the end
  write   tokens, spare slots (-1) at the end, heads, page size
  paged   batch, own lengths, query lengths, prefix length, heads, page size,
          softcap (0: none), slopes (whether scores fall with distance), lse
  scored  schedule kind, packed lengths, heads, tile, sections, softcap,
          slopes, lse
Lengths are drawn log-uniformly between two bounds from ``lens``, a seed that
belongs to the case, so that the work of a case is known without its tensors.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"


def _map(name, batch, cached, new, page, spare, lens=1):
    return {"name": name, "op": "map", "batch": batch, "cached_lo": cached[0],
            "cached_hi": cached[1], "new_lo": new[0], "new_hi": new[1], "page": page,
            "spare": spare, "lens": lens}


def _write(name, tokens, spare, hq, hkv, d, page):
    return {"name": name, "op": "write", "tokens": tokens, "spare": spare, "hq": hq, "hkv": hkv,
            "d": d, "page": page}


def _paged(name, batch, own_lens, q_lens, prefix, hq, hkv, d, page, softcap=0.0, slopes=False,
           lse=False, lens=1):
    return {"name": name, "op": "paged", "batch": batch, "own_lo": own_lens[0],
            "own_hi": own_lens[1], "q_lo": q_lens[0], "q_hi": q_lens[1], "prefix": prefix,
            "hq": hq, "hkv": hkv, "d": d, "page": page, "softcap": softcap, "slopes": slopes,
            "lse": lse, "lens": lens}


def _scored(name, kind, lens, hq, hkv, d, tile, sink=0, window=1, last=0, softcap=0.0,
            slopes=False, lse=False):
    return {"name": name, "op": "scored", "kind": kind, "lens": ",".join(str(n) for n in lens),
            "hq": hq, "hkv": hkv, "d": d, "tile": tile, "sink": sink, "window": window,
            "last": last, "softcap": softcap, "slopes": slopes, "lse": lse}


def listed():
    return [
        # one decode step of a full server: 64 requests, a token each
        _map("map_decode_64", 64, (100, 16000), (1, 1), 16, 0),
        # a wave of long prompts beside running requests: about half a million
        # new tokens in ragged pieces, spare slots at the end as a captured
        # graph keeps them
        _map("map_prompts_192", 192, (1, 30000), (1, 24000), 16, 5000),
        # the cache write of a decode step, from the rows of a fused projection
        _write("write_decode_64", 64, 0, 32, 8, 128, 16),
        # the cache write of a 64K-token prefill layer
        _write("write_prefill_64k", 65536, 77, 32, 8, 128, 64),
        # the smallest attention call: one request, 1024 tokens, one kv head
        _paged("paged_tiny_1k_d64", 1, (1024, 1024), (1, 1), 0, 4, 1, 64, 16),
        # an ordinary decode step: 64 ragged requests
        _paged("paged_decode_64", 64, (200, 12000), (1, 1), 0, 32, 8, 128, 16, lse=True),
        # a batch behind one long system prompt whose end is inside a page
        _paged("paged_prefix_128", 128, (17, 1500), (1, 1), 12345, 32, 8, 128, 16),
        # the largest caches: four requests of 128K, seven heads to a kv head
        _paged("paged_long_4_g7", 4, (131072, 131072), (1, 1), 0, 28, 4, 128, 64),
        # drafted tokens of a model with capped scores and a prefix
        _paged("paged_draft_cap", 24, (300, 9000), (1, 6), 2048, 32, 4, 64, 32, softcap=30.0,
               slopes=True, lse=True),
        # the next pieces of four prompts against their caches
        _paged("paged_chunk_4", 4, (4000, 16000), (700, 2048), 0, 32, 8, 128, 64, softcap=50.0),
        # prefill of a model with capped scores: a dense layer
        _scored("scored_causal_16k_cap", "causal", [16384], 32, 8, 128, 128, softcap=50.0,
                lse=True),
        # a Triangle layer of a model whose scores fall with distance, packed
        # ragged prompts
        _scored("scored_tri_packed_bias", "triangle", [24001, 317, 1, 15360, 2990, 129], 32, 8,
                128, 128, 128, 2048, 128, slopes=True),
    ]


_LARGEST = 2.2e12  # flops of the largest drawn case (the largest listed one has 2.2e12)


def draw(rng):
    """One more case of the same ranges."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    span = lambda lo, hi: sorted((log(lo, hi), log(lo, hi)))  # noqa: E731
    while True:
        op = rng.choices(["map", "write", "paged", "scored"], [2, 2, 6, 4])[0]
        d = rng.choice([128, 128, 64])
        group = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8])
        hkv = rng.choice([1, 2, 4, 8, 8])
        page = rng.choice([16, 16, 32, 64, 128])
        if op == "map":
            batch = log(1, 1000)
            top = max(2, 600000 // batch)
            c = _map(None, batch, span(1, 40000),
                     rng.choice([(1, 1), span(1, min(40000, top))]), page,
                     rng.choice([0, log(1, 5000)]), rng.randrange(1 << 30))
        elif op == "write":
            c = _write(None, log(1, 65536), rng.choice([0, log(1, 500)]), group * hkv, hkv, d,
                       page)
        elif op == "paged":
            q = rng.choice([(1, 1), (1, 1), (1, rng.randrange(2, 9)), span(1, 1500)])
            c = _paged(None, log(1, 256), span(q[1], 131072), q,
                       rng.choice([0, 0, log(1, 32768)]), group * hkv, hkv, d, page,
                       rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]), rng.random() < 0.3,
                       rng.random() < 0.5, rng.randrange(1 << 30))
            # what the caches of a case may hold
            if c["batch"] * (c["own_hi"] + c["prefix"]) > 800000 or c["batch"] * q[1] > 20000 \
                    or c["batch"] * q[1] * c["hq"] * (c["own_hi"] + c["prefix"]) > 2e9:
                continue
        else:
            kind = rng.choice(["triangle", "triangle", "causal"])
            total = log(100, 49152 if kind == "triangle" else 16384)
            lens = [total]
            if rng.random() < 0.4:  # a packed batch
                cuts = sorted(rng.randrange(total + 1) for _ in range(rng.randrange(1, 8)))
                lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
            cap = rng.choice([0.0, 15.0, 30.0, 50.0])
            tri = kind == "triangle"
            c = _scored(None, kind, lens, group * hkv, hkv, d, rng.choice([64, 128, 128]),
                        rng.choice([0, 8, 64, 128, rng.randrange(1, 257)]) if tri else 0,
                        rng.choice([512, 2048, log(64, 4096)]) if tri else 1,
                        rng.choice([0, 64, 128, rng.randrange(1, 257)]) if tri else 0, cap,
                        cap == 0.0 or rng.random() < 0.3, rng.random() < 0.5)
        del c["name"]
        if work(c)["flops"] <= _LARGEST:
            return c


# ---------------------------------------------------------------- lengths
def _draws(case, n, lo, hi, salt):
    rng = random.Random(case["lens"] * 16 + salt)
    return [int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) for _ in range(n)]


def _map_lens(case):
    return (_draws(case, case["batch"], case["cached_lo"], case["cached_hi"], 1),
            _draws(case, case["batch"], case["new_lo"], case["new_hi"], 2))


def _paged_lens(case):
    """Own keys (this call's tokens among them) and query rows a request."""
    q = _draws(case, case["batch"], case["q_lo"], case["q_hi"], 2)
    kv = _draws(case, case["batch"], case["own_lo"], case["own_hi"], 1)
    return [max(a, b) for a, b in zip(kv, q)], q


def _packed(case):
    return [int(x) for x in case["lens"].split(",")]


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _pages(n, page):
    return -(-n // page)


# ----------------------------------------------------------------- inputs
def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _slopes(case):
    # a geometric sequence over the heads, as such models use
    h = torch.arange(1, case["hq"] + 1, dtype=torch.float32, device=DEVICE)
    return torch.exp2(-8.0 * h / case["hq"]) if case["slopes"] else None


def _tables(lens, page, g, spare_pages=5):
    """A table of pages in random order for requests of these lengths; -1
    where a request has none.  Returns the table and the pages left."""
    need = [_pages(n, page) for n in lens]
    total, width = sum(need), max(need + [1]) + 2
    order = torch.randperm(total + spare_pages, generator=g, device=DEVICE).to(torch.int32)
    used = torch.arange(width, device=DEVICE)[None, :] < _ints(need)[:, None]
    at = torch.cumsum(used.flatten(), 0).view(used.shape) - 1
    table = torch.where(used, order[at.clamp(0, total + spare_pages - 1)], -1)
    return table.to(torch.int32).contiguous(), order[total:].contiguous(), total + spare_pages


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE).bfloat16()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = {"case": case}
    if case["op"] == "map":
        cached, new = _map_lens(case)
        page = case["page"]
        kv = [a + b for a, b in zip(cached, new)]
        table, _, n_pages = _tables(cached, page, g)
        width = max(_pages(n, page) for n in kv) + 3
        wide = torch.full((case["batch"], width), -1, dtype=torch.int32, device=DEVICE)
        w = min(width, table.shape[1])
        wide[:, :w] = table[:, :w]
        fresh = sum(_pages(a, page) - _pages(b, page) for a, b in zip(kv, cached)) + 9
        free = torch.randperm(fresh, generator=g, device=DEVICE).to(torch.int32) + n_pages
        count = sum(new) + case["spare"]
        s.update(cached=_ints(cached), new=_ints(new), table=wide, free=free,
                 n_free=_ints([fresh - 4]), kv=torch.empty_like(_ints(kv)),
                 cu=torch.empty(case["batch"] + 1, dtype=torch.int32, device=DEVICE),
                 slots=torch.empty(count, dtype=torch.int32, device=DEVICE),
                 state=torch.empty(2, dtype=torch.int32, device=DEVICE))
        return s
    if case["op"] == "write":
        n, hq, hkv, d, page = (case[x] for x in ("tokens", "hq", "hkv", "d", "page"))
        rows = n + case["spare"]
        qkv = _normal(g, rows, hq + 2 * hkv, d)  # a fused projection's output
        pages = _pages(n, page) + 3
        slots = torch.full((rows,), -1, dtype=torch.int32, device=DEVICE)
        base = torch.randperm(pages, generator=g, device=DEVICE)
        tok = torch.arange(n, device=DEVICE)
        slots[:n] = (base[tok // page] * page + tok % page).to(torch.int32)
        s.update(k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], slots=slots,
                 k_cache=_normal(g, pages, hkv, page, d), v_cache=_normal(g, pages, hkv, page, d))
        return s
    if case["op"] == "paged":
        kv, q_lens = _paged_lens(case)
        hq, hkv, d, page, prefix = (case[x] for x in ("hq", "hkv", "d", "page", "prefix"))
        table, left, n_pages = _tables(kv, page, g, _pages(prefix, page) + 3)
        s.update(kv_host=kv, q_host=q_lens, total=sum(q_lens), kv=_ints(kv), table=table,
                 cu_q=None if max(q_lens) == 1 else _ints(_offsets(q_lens)),
                 prefix_pages=left[:_pages(prefix, page)].contiguous() if prefix else None,
                 q=_normal(g, sum(q_lens), hq, d), slopes=_slopes(case))
        s["k_cache"] = _normal(g, n_pages, hkv, page, d)
        s["v_cache"] = _normal(g, n_pages, hkv, page, d)
        # an attention sink, as cases of the prefill passes have it; the
        # places behind a request's last token hold what was there before
        first = s["prefix_pages"][:1] if prefix else table[:, 0].clamp(min=0)
        s["k_cache"][first.long(), :, 0] *= 8.0
        last, end = (s["kv"].long() - 1) // page, s["kv"].long() % page
        tail = table.gather(1, last[:, None])[:, 0].long()
        behind = (torch.arange(page, device=DEVICE)[None, :] >= end[:, None]) & (end > 0)[:, None]
        for x in (s["k_cache"], s["v_cache"]):
            x[tail] = x[tail].masked_fill(behind[:, None, :, None], math.nan)
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = (torch.empty(hq, s["total"], dtype=torch.float32, device=DEVICE)
                    if case["lse"] else None)
        if own:
            from paper_2507_21526_amd import binding
            s["plan"] = binding.PagedPlan(case["batch"], s["total"], hq, hkv, d,
                                          prefix=prefix > 0, ragged=s["cu_q"] is not None)
        return s
    lens = _packed(case)
    total, hq, hkv, d = sum(lens), case["hq"], case["hkv"], case["d"]
    k = torch.randn(total, hkv, d, generator=g, device=DEVICE)
    first = [b for b, n in zip(_offsets(lens), lens) if n]
    k[first] *= 8.0
    s.update(q=_normal(g, total, hq, d), k=k.bfloat16(), v=_normal(g, total, hkv, d),
             slopes=_slopes(case), cu=_offsets(lens))
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = (torch.empty(hq, total, dtype=torch.float32, device=DEVICE)
                if case["lse"] else None)
    if own:
        from paper_2507_21526_amd import binding
        s["plan"] = binding.Plan(case["kind"], s["cu"], case["sink"], case["window"],
                                 case["last"], case["tile"], hq, d)
    return s


# -------------------------------------------------------------- one pass
def run(state):
    s, case = state, state["case"]
    if own:
        return _run_own(s, case)
    return {"map": _plain_map, "write": _plain_write, "paged": _plain_paged,
            "scored": _plain_scored}[case["op"]](s, case)


def _run_own(s, case):
    from paper_2507_21526_amd import binding
    cap = case.get("softcap") or None
    if case["op"] == "map":
        binding.page_map(s["cached"], s["new"], s["table"], s["free"], s["n_free"], case["page"],
                         s["kv"], s["cu"], s["slots"], s["state"])
        return {"table": s["table"], "kv": s["kv"], "cu": s["cu"], "slots": s["slots"],
                "state": s["state"]}
    if case["op"] == "write":
        binding.kv_cache_write(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
        return {"k": s["k_cache"], "v": s["v_cache"]}
    if case["op"] == "paged":
        s["plan"].run(s["q"], s["k_cache"], s["v_cache"], s["o"], s["kv"], s["table"],
                      cu_q=s["cu_q"], prefix_pages=s["prefix_pages"], prefix_len=case["prefix"],
                      lse=s["lse"], softcap=cap, slopes=s["slopes"])
    else:
        s["plan"].run(s["q"], s["k"], s["v"], s["o"], s["lse"], softcap=cap, slopes=s["slopes"])
    return {"o": s["o"], "lse": s["lse"]}


def _plain_map(s, case):
    page = case["page"]
    table, free, cached, new = s["table"], s["free"].long(), s["cached"].long(), s["new"].long()
    width, count = table.shape[1], s["slots"].numel()
    n_free = s["n_free"].long()
    kv = cached + new
    had = (cached + page - 1) // page
    need = (kv + page - 1) // page - had
    cu = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0))
    first = torch.cumsum(need, 0) - need  # rank of a request's first new page
    # new pages come from the end of the free list, in the requests' order
    x = torch.arange(width, device=DEVICE)[None, :]
    rank = first[:, None] + x - had[:, None]
    fresh = free[(n_free - 1 - rank).clamp(0, free.numel() - 1)].to(torch.int32)
    table.copy_(torch.where((x >= had[:, None]) & (x < (had + need)[:, None]), fresh, table))
    tok = torch.arange(count, device=DEVICE)
    b = torch.searchsorted(cu[1:], tok, right=True).clamp(max=case["batch"] - 1)
    pos = cached[b] + tok - cu[b]
    at = table[b, (pos // page).clamp(max=width - 1)].long() * page + pos % page
    slots = torch.where(tok < cu[-1], at, -1)
    state = torch.cat([n_free - need.sum(), torch.zeros_like(n_free)])
    return {"table": table, "kv": kv.to(torch.int32), "cu": cu.to(torch.int32),
            "slots": slots.to(torch.int32), "state": state.to(torch.int32)}


def _plain_write(s, case):
    n, page = case["tokens"], case["page"]
    at = s["slots"][:n].long()
    s["k_cache"][at // page, :, at % page] = s["k"][:n]
    s["v_cache"][at // page, :, at % page] = s["v"][:n]
    return {"k": s["k_cache"], "v": s["v_cache"]}


def _scores(case, slopes, x, distance):
    """Scaled products [.., heads, rows, keys] in place to scores; distance
    from key to row [.., 1, rows, keys]."""
    if case["softcap"]:
        x.div_(case["softcap"]).tanh_().mul_(case["softcap"])
    if slopes is not None:
        x.sub_(slopes[:, None, None] * distance)
    return x


def _softmax(x, keep):
    """(probabilities, log-sum-exp) of scores over the kept keys; zeros and
    -inf for a row that keeps none."""
    x.masked_fill_(~keep, -math.inf)
    top = x.amax(-1, keepdim=True)
    top.masked_fill_(top == -math.inf, 0.0)
    p = x.sub_(top).exp_()
    den = p.sum(-1, keepdim=True)
    lse = torch.where(den > 0, top + den.log(), -math.inf)[..., 0]
    return p.div_(den.clamp(min=1e-38)), lse


def _plain_paged(s, case):
    hq, hkv, d, page, prefix, batch = (case[x] for x in ("hq", "hkv", "d", "page", "prefix",
                                                         "batch"))
    group, rows, keys = hq // hkv, max(s["q_host"]), max(s["kv_host"])
    cu = s["cu_q"].long() if s["cu_q"] is not None else torch.arange(batch + 1, device=DEVICE)
    kv = s["kv"].long()
    # padded queries [batch, hkv, group * rows, d]
    t = torch.arange(rows, device=DEVICE)
    n_q = cu[1:] - cu[:-1]
    tok = (cu[:-1, None] + t).clamp(max=s["total"] - 1)
    q = s["q"][tok].float() * d ** -0.5
    q = q.view(batch, rows, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(batch, hkv,
                                                                          group * rows, d)
    # padded own keys and values [batch, hkv, keys, d], zero behind the last
    j = torch.arange(keys, device=DEVICE)
    live = j < kv[:, None]
    pages = s["table"][:, :_pages(keys, page)].clamp(min=0).long()

    def padded(cache):
        x = cache[pages].float().transpose(1, 2).reshape(batch, hkv, -1, d)[:, :, :keys]
        return torch.where(live[:, None, :, None], x, 0.0)

    pos = kv[:, None] - n_q[:, None] + t
    dist = (pos[:, :, None] - j).float()[:, None]  # [batch, 1, rows, keys]
    keep = (dist >= 0) & live[:, None, None]
    k, v = padded(s["k_cache"]), padded(s["v_cache"])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(batch, hq, rows, keys)
    x = _scores(case, s["slopes"], x, dist)
    if prefix:  # the prefix's keys come before every request's own
        def shared(cache):
            y = cache[s["prefix_pages"].long()].float().transpose(0, 1)
            return y.reshape(hkv, -1, d)[:, :prefix]

        kp, vp = shared(s["k_cache"]), shared(s["v_cache"])
        qp = q.transpose(0, 1).reshape(hkv, -1, d)
        y = torch.matmul(qp, kp.transpose(1, 2).contiguous())
        y = y.view(hkv, batch, group, rows, prefix).transpose(0, 1)
        y = y.reshape(batch, hq, rows, prefix)
        far = (pos[:, :, None] + prefix - torch.arange(prefix, device=DEVICE)).float()[:, None]
        y = _scores(case, s["slopes"], y, far)
        x = torch.cat([y, x], -1)
        keep = torch.cat([(pos >= 0)[:, None, :, None].expand(-1, -1, -1, prefix), keep], -1)
    p, lse = _softmax(x, keep)
    own_p = p[..., prefix:].reshape(batch, hkv, group * rows, keys)
    o = torch.matmul(own_p, v).view(batch, hq, rows, d)
    if prefix:
        pp = p[..., :prefix].reshape(batch, hkv, group * rows, prefix).transpose(0, 1)
        op = torch.matmul(pp.reshape(hkv, -1, prefix), vp)
        o += op.view(hkv, batch, group, rows, d).transpose(0, 1).reshape(batch, hq, rows, d)
    # back to packed rows
    r = torch.arange(s["total"], device=DEVICE)
    b = torch.searchsorted(cu[1:], r, right=True)
    o, lse = o[b, :, r - cu[b]], lse[b, :, r - cu[b]]
    return {"o": o.bfloat16(), "lse": lse.t().contiguous() if case["lse"] else None}


def _row_blocks(case):
    """(offset, r0, r1, sequence length, streaming) blocks of rows whose
    scores fit in memory: Last and dense rows see every earlier key,
    streaming ones the sink and a window."""
    blocks = []
    for off, n in zip(_offsets(_packed(case)), _packed(case)):
        first_last = n - min(case["last"], n) if case["kind"] == "triangle" else 0
        r0 = 0
        while r0 < n:
            streaming = r0 < first_last
            r1 = min(r0 + (2048 if streaming else 1024), first_last if streaming else n)
            blocks.append((off, r0, r1, streaming))
            r0 = r1
    return blocks


def _plain_scored(s, case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, total = hq // hkv, s["q"].shape[0]
    o = torch.empty(total, hq, d, dtype=torch.float32, device=DEVICE)
    lse = torch.empty(hq, total, dtype=torch.float32, device=DEVICE)
    for off, r0, r1, streaming in _row_blocks(case):
        lo = max(0, r0 - case["window"] + 1) if streaming else 0
        n_sink = min(case["sink"], lo)
        at = torch.cat([torch.arange(n_sink, device=DEVICE), torch.arange(lo, r1, device=DEVICE)])
        dist = torch.arange(r0, r1, device=DEVICE)[:, None] - at
        keep = dist >= 0
        if streaming:
            keep &= (dist < case["window"]) | (at < case["sink"])
        q = s["q"][off + r0:off + r1].float().mul_(d ** -0.5)
        q = q.view(r1 - r0, hkv, group, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
        k = s["k"][off + at].float().permute(1, 2, 0).contiguous()
        x = torch.matmul(q, k).view(hq, r1 - r0, -1)
        p, lse[:, off + r0:off + r1] = _softmax(_scores(case, s["slopes"], x, dist.float()), keep)
        v = s["v"][off + at].float().transpose(0, 1).contiguous()
        y = torch.matmul(p.view(hkv, group * (r1 - r0), -1), v)
        o[off + r0:off + r1] = y.view(hq, r1 - r0, d).transpose(0, 1)
    return {"o": o.bfloat16(), "lse": lse if case["lse"] else None}


# ------------------------------------------------------------------- work
def _map_work(case):
    cached, new = _map_lens(case)
    page = case["page"]
    fresh = sum(_pages(a + b, page) - _pages(a, page) for a, b in zip(cached, new))
    # lengths in and out, free pages read, entries written, one open page a
    # request read, slots written
    nbytes = 4 * (3 * case["batch"] + case["batch"] + 1 + 2 * fresh + case["batch"] + 3 +
                  sum(new) + case["spare"])
    return {"bytes": nbytes, "flops": 0}


def _paged_work(case):
    kv, q = _paged_lens(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pairs = sum(b * (a + case["prefix"]) - b * (b - 1) // 2 for a, b in zip(kv, q))
    nbytes = 2 * 2 * hkv * d * (sum(kv) + case["prefix"]) + 2 * 2 * sum(q) * hq * d
    nbytes += 4 * sum(_pages(n, case["page"]) for n in kv) + 8 * case["batch"]
    nbytes += 4 * hq * sum(q) if case["lse"] else 0
    return {"bytes": nbytes, "flops": 4 * d * hq * pairs}


def _scored_work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pairs = 0
    for n in _packed(case):
        first_last = n - min(case["last"], n) if case["kind"] == "triangle" else 0
        pairs += (first_last + 1 + n) * (n - first_last) // 2
        w, sk = case["window"], case["sink"]
        m = min(first_last, w)
        pairs += m * (m + 1) // 2 + (first_last - m) * w
        # sink keys before the window of row i: min(sink, i + 1 - w)
        out = max(0, first_last - w)
        short = min(out, sk)
        pairs += short * (short + 1) // 2 + (out - short) * sk
    total = sum(_packed(case))
    nbytes = 2 * total * (2 * hq + 2 * hkv) * d + (4 * total * hq if case["lse"] else 0)
    return {"bytes": nbytes, "flops": 4 * d * hq * pairs}


def work(case):
    """Each input read and each output written once; two contractions per
    kept (row, key) pair."""
    if case["op"] == "map":
        return _map_work(case)
    if case["op"] == "write":
        n, hkv, d = case["tokens"], case["hkv"], case["d"]
        return {"bytes": 8 * n * hkv * d + 4 * (n + case["spare"]), "flops": 0}
    return _paged_work(case) if case["op"] == "paged" else _scored_work(case)


# ------------------------------------------------------------ 64-bit form
def _rows64(q, k, v, keep, dist, case, slope):
    """One head's rows [r, d] over keys [n, d] in 64 bits: (o, lse)."""
    x = (q @ k.t().contiguous()) / math.sqrt(case["d"])
    if case["softcap"]:
        x = case["softcap"] * torch.tanh(x / case["softcap"])
    if slope is not None:
        x = x - float(slope) * dist
    x = torch.where(keep, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, -1)
    p = torch.where(keep, torch.exp(x - lse[:, None]), torch.zeros_like(x))
    return p @ v, lse


def exact(case, seed):
    if case["op"] == "map":
        return None  # integers
    if case["op"] == "write":
        return _exact_write(case, seed)
    if case["op"] == "paged":
        return _exact_paged(case, seed)
    return _exact_scored(case, seed)


def _exact_write(case, seed):
    """Every head of every token to its place, a page's places laid out as
    one axis."""
    s = prepare(case, seed)
    at = s["slots"][:case["tokens"]].long()
    out = {}
    for name in ("k", "v"):
        pages, hkv, page, d = s[name + "_cache"].shape
        flat = s[name + "_cache"].to(torch.float64).transpose(1, 2).reshape(-1, hkv, d)
        flat.index_copy_(0, at, s[name][:case["tokens"]].to(torch.float64))
        out[name] = flat.view(pages, page, hkv, d).transpose(1, 2).contiguous()
    return out


def _exact_paged(case, seed):
    s = prepare(case, seed)
    hq, hkv, d, page, prefix = (case[x] for x in ("hq", "hkv", "d", "page", "prefix"))
    if work(case)["flops"] > 3e12 or case["batch"] * hq > 20000:
        return None
    o = torch.zeros(s["total"], hq, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((hq, s["total"]), -math.inf, dtype=torch.float64, device=DEVICE)
    start = 0
    for b, (n, m) in enumerate(zip(s["kv_host"], s["q_host"])):
        at = torch.arange(prefix + n, device=DEVICE)
        mine = torch.arange(n, device=DEVICE)
        page_of = s["table"][b].long()[mine // page]
        place = mine % page
        if prefix:
            pre = torch.arange(prefix, device=DEVICE)
            page_of = torch.cat([s["prefix_pages"].long()[pre // page], page_of])
            place = torch.cat([pre % page, place])
        for r0 in range(0, m, 512):
            r1 = min(m, r0 + 512)
            row = prefix + n - m + torch.arange(r0, r1, device=DEVICE)
            dist = (row[:, None] - at).to(torch.float64)
            for g in range(hkv):
                k = s["k_cache"][page_of, g, place].to(torch.float64)
                v = s["v_cache"][page_of, g, place].to(torch.float64)
                for h in range(g * (hq // hkv), (g + 1) * (hq // hkv)):
                    q = s["q"][start + r0:start + r1, h].to(torch.float64)
                    a, e = _rows64(q, k, v, dist >= 0, dist, case,
                                   None if s["slopes"] is None else s["slopes"][h].item())
                    o[start + r0:start + r1, h], lse[h, start + r0:start + r1] = a, e
        start += m
    return {"o": o, "lse": lse if case["lse"] else None}


def _exact_scored(case, seed):
    s = prepare(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    total = s["q"].shape[0]
    o = torch.zeros(total, hq, d, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(hq, total, dtype=torch.float64, device=DEVICE)
    triangle = case["kind"] == "triangle"
    for off, n in zip(s["cu"], _packed(case)):
        last0 = n - min(case["last"], n)
        edges = sorted({0, n, last0, *range(0, n, 4096)})
        for r0, r1 in zip(edges, edges[1:]):
            row = torch.arange(r0, r1, device=DEVICE)[:, None]
            stream = triangle and r0 < last0
            near = max(0, r0 - case["window"] + 1) if stream else 0
            key = torch.arange(r1, device=DEVICE)
            key = key[(key < case["sink"]) | (key >= near)] if stream else key
            gap = row - key
            keep = gap >= 0
            if stream:
                keep = keep & ((gap < case["window"]) | (key < case["sink"]))
            for h in range(hq):
                kv = h // (hq // hkv)
                a, e = _rows64(s["q"][off + r0:off + r1, h].to(torch.float64),
                               s["k"][off + key, kv].to(torch.float64),
                               s["v"][off + key, kv].to(torch.float64), keep,
                               gap.to(torch.float64), case,
                               None if s["slopes"] is None else s["slopes"][h].item())
                o[off + r0:off + r1, h], lse[h, off + r0:off + r1] = a, e
    return {"o": o, "lse": lse if case["lse"] else None}
