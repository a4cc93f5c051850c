"""Performance cases of the 8-bit paged cache: rows of new tokens quantised into
their slots, cached rows read back as bf16, and attention over the cache.

A case is one call that a serving program makes for one layer: ``write`` and
``paged`` in every step, ``read`` when a prefill needs keys and values that are
already cached.  With ``own`` set, ``run`` makes the framework's call; without
it, the same result is computed from elementary torch operations in fp32.

The 8-bit form.  A row is what one kv head holds of one token, head_dim
elements.  It is held as e4m3 elements and one scale 2^e, e the least integer
of at least -100 for which no finite element of the row passes 448 2^e; an
element is x 2^-e rounded to the nearest e4m3 value (ties to the even one; 240
is the largest where e = 120, so that what comes back is finite), and NaN where
x is infinite or NaN.

Fields of a case (beside name and op)
  write   tokens, spare slots (-1) at the end, heads, page size
  read    form of the cache (8 bits or bf16), batch, rows read a request,
          positions skipped before them, spare rows at the end, heads, page size
  paged   batch, own lengths, query lengths, prefix length, heads, page size,
          softcap (0: none), slopes (whether scores fall with distance), lse
Lengths are drawn log-uniformly between two bounds from ``lens``, a seed that
belongs to the case, so that the work of a case is known without its tensors.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
LEAST_E, MOST_E = -100, 120  # of a scale 2^e


def _write(name, tokens, spare, hq, hkv, d, page):
    return {"name": name, "op": "write", "tokens": tokens, "spare": spare, "hq": hq, "hkv": hkv,
            "d": d, "page": page}


def _read(name, form, batch, rows, skip, spare, hkv, d, page, lens=1):
    return {"name": name, "op": "read", "form": form, "batch": batch, "rows_lo": rows[0],
            "rows_hi": rows[1], "skip_lo": skip[0], "skip_hi": skip[1], "spare": spare,
            "hkv": hkv, "d": d, "page": page, "lens": lens}


def _paged(name, batch, own_lens, q_lens, prefix, hq, hkv, d, page, softcap=0.0, slopes=False,
           lse=False, lens=1):
    return {"name": name, "op": "paged", "batch": batch, "own_lo": own_lens[0],
            "own_hi": own_lens[1], "q_lo": q_lens[0], "q_hi": q_lens[1], "prefix": prefix,
            "hq": hq, "hkv": hkv, "d": d, "page": page, "softcap": softcap, "slopes": slopes,
            "lse": lse, "lens": lens}


def listed():
    return [
        # the cache write of a decode step, from the rows of a fused projection
        _write("write8_decode_96", 96, 0, 32, 8, 128, 16),
        # the cache write of a piece of a prompt, an odd number of tokens
        _write("write8_piece_5001_d64", 5001, 15, 28, 4, 64, 32),
        # the cache write of a 64K-token prefill layer
        _write("write8_prefill_64k", 65536, 77, 32, 8, 128, 64),
        # one cached prompt read back for a prefill that attends to it
        _read("read8_prompt_20011", "8bit", 1, (20011, 20011), (0, 0), 0, 8, 128, 16),
        # the ends of a batch's cached prompts, from inside a page on
        _read("read8_batch_48_d64", "8bit", 48, (1, 3000), (1, 9000), 100, 4, 64, 32),
        # the same call on a cache that holds bf16: four prompts, 64K rows
        _read("read16_prompts_64k", "bf16", 4, (16384, 16384), (0, 0), 0, 8, 128, 64),
        # the smallest attention call: one request, one kv head
        _paged("paged8_tiny_700_d64", 1, (700, 700), (1, 1), 0, 4, 1, 64, 16),
        # an ordinary decode step: 96 ragged requests
        _paged("paged8_decode_96", 96, (150, 15000), (1, 1), 0, 32, 8, 128, 16, lse=True),
        # a batch behind one long system prompt whose end is inside a page
        _paged("paged8_prefix_160", 160, (9, 1200), (1, 1), 10007, 32, 8, 128, 32),
        # the largest caches: three requests of 128K, seven heads to a kv head
        _paged("paged8_long_3_g7", 3, (131072, 131072), (1, 1), 0, 28, 4, 128, 64),
        # drafted tokens of a model with capped and biased scores, and a prefix
        _paged("paged8_draft_cap_d64", 24, (300, 9000), (1, 6), 2048, 32, 4, 64, 32,
               softcap=30.0, slopes=True, lse=True),
        # the next pieces of five prompts against their caches
        _paged("paged8_chunk_5", 5, (3000, 15000), (500, 1800), 0, 32, 8, 128, 64),
    ]


_MOST_FLOPS = 6.3e11  # of a drawn case (paged8_chunk_5 has 6.4e11)
_MOST_ROWS = 366000   # keys of all requests of a drawn case (paged8_decode_96 holds 366700)


def draw(rng):
    """One more case of the same ranges."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    span = lambda lo, hi: sorted((log(lo, hi), log(lo, hi)))  # noqa: E731
    while True:
        op = rng.choices(["write", "read", "paged"], [3, 3, 7])[0]
        d = rng.choice([128, 128, 64])
        group = rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8])
        hkv = rng.choice([1, 2, 4, 8, 8])
        page = rng.choice([16, 16, 32, 64, 128, 256])
        if op == "write":
            c = _write(None, log(1, 65536), rng.choice([0, log(1, 500)]), group * hkv, hkv, d,
                       page)
        elif op == "read":
            batch = log(1, 300)
            c = _read(None, rng.choice(["8bit", "8bit", "bf16"]), batch,
                      span(1, max(2, 65536 // batch)), rng.choice([(0, 0), span(1, 5000)]),
                      rng.choice([0, log(1, 500)]), hkv, d, page, rng.randrange(1 << 30))
            if batch * (c["rows_hi"] + c["skip_hi"]) > _MOST_ROWS:
                continue
        else:
            q = rng.choice([(1, 1), (1, 1), (1, rng.randrange(2, 9)), span(1, 1500)])
            c = _paged(None, log(1, 256), span(q[1], 131072), q,
                       rng.choice([0, 0, log(1, 32768)]), group * hkv, hkv, d, page,
                       rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]), rng.random() < 0.3,
                       rng.random() < 0.5, rng.randrange(1 << 30))
            keys = c["own_hi"] + c["prefix"]
            # what the plain form's padded scores may take
            if c["batch"] * keys > _MOST_ROWS or c["batch"] * q[1] > 20000 \
                    or c["batch"] * q[1] * c["hq"] * keys > 2e9:
                continue
        del c["name"]
        if work(c)["flops"] <= _MOST_FLOPS:
            return c


# ---------------------------------------------------------------- lengths
def _draws(case, n, lo, hi, salt):
    if lo == hi:
        return [lo] * n
    rng = random.Random(case["lens"] * 16 + salt)
    return [int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) for _ in range(n)]


def _read_lens(case):
    """Rows read and positions skipped a request."""
    return (_draws(case, case["batch"], case["rows_lo"], case["rows_hi"], 1),
            _draws(case, case["batch"], case["skip_lo"], case["skip_hi"], 2))


def _paged_lens(case):
    """Own keys (this call's tokens among them) and query rows a request."""
    q = _draws(case, case["batch"], case["q_lo"], case["q_hi"], 2)
    kv = _draws(case, case["batch"], case["own_lo"], case["own_hi"], 1)
    return [max(a, b) for a, b in zip(kv, q)], q


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _pages(n, page):
    return -(-n // page)


# ----------------------------------------------------------- the 8-bit form
def _pow2(e):
    """2^e of int32 e in -126 .. 127, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows [..., d] as (e4m3 [..., d], scales e8m0 [...])."""
    x = x.float()
    fine = torch.isfinite(x)
    top = torch.where(fine, x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = torch.where(top > 0, e - 9 + (m > 0.875).int(), LEAST_E).clamp(min=LEAST_E).int()
    most = torch.where(e == MOST_E, 240.0, 448.0)[..., None]
    y = torch.minimum(torch.maximum(x * _pow2(-e)[..., None], -most), most)
    y = torch.where(fine, y, math.nan).to(torch.float8_e4m3fn)
    return y, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _scale(s):
    """fp32 values of e8m0 scales (bytes 1 .. 254; others do not reach a result)."""
    return _pow2(s.view(torch.uint8).int() - 127)


def _taken(x, at):
    """x[at] of an 8-bit tensor."""
    return x.view(torch.uint8)[at].view(x.dtype)


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


def _keys(g, pages, hkv, page, d):
    """Keys whose channels differ in size, as keys of trained models do."""
    size = torch.exp(0.5 * torch.randn(hkv, 1, d, generator=g, device=DEVICE)).clamp(max=3.0)
    return _normal(g, pages, hkv, page, d) * size.bfloat16()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = {"case": case}
    hkv, d, page = case["hkv"], case["d"], case["page"]
    if case["op"] == "write":
        n, hq = case["tokens"], case["hq"]
        rows = n + case["spare"]
        qkv = _normal(g, rows, hq + 2 * hkv, d)  # a fused projection's output
        pages = _pages(n, page) + 3
        slots = torch.full((rows,), -1, dtype=torch.int32, device=DEVICE)
        base = torch.randperm(pages, generator=g, device=DEVICE)
        tok = torch.arange(n, device=DEVICE)
        slots[:n] = (base[tok // page] * page + tok % page).to(torch.int32)
        s.update(k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], slots=slots)
        s["k_cache"], s["k_scale"] = _quantise(_keys(g, pages, hkv, page, d))
        s["v_cache"], s["v_scale"] = _quantise(_normal(g, pages, hkv, page, d))
        return s
    if case["op"] == "read":
        rows, skip = _read_lens(case)
        cu = _offsets(rows)
        table, _, n_pages = _tables([a + b for a, b in zip(rows, skip)], page, g)
        k, v = _keys(g, n_pages, hkv, page, d), _normal(g, n_pages, hkv, page, d)
        s.update(table=table, cu=_ints(cu), starts=_ints(skip) if case["skip_hi"] else None,
                 total=cu[-1], k_cache=k, v_cache=v, k_scale=None, v_scale=None)
        if case["form"] == "8bit":
            s["k_cache"], s["k_scale"] = _quantise(k)
            s["v_cache"], s["v_scale"] = _quantise(v)
        s["k"] = _normal(g, cu[-1] + case["spare"], hkv, d)
        s["v"] = _normal(g, cu[-1] + case["spare"], hkv, d)
        return s
    kv, q_lens = _paged_lens(case)
    hq, prefix = case["hq"], case["prefix"]
    table, left, n_pages = _tables(kv, page, g, _pages(prefix, page) + 3)
    s.update(kv_host=kv, q_host=q_lens, total=sum(q_lens), kv=_ints(kv), table=table,
             cu_q=None if max(q_lens) == 1 else _ints(_offsets(q_lens)),
             prefix_pages=left[:_pages(prefix, page)].contiguous() if prefix else None,
             q=_normal(g, sum(q_lens), hq, d), slopes=_slopes(case))
    k = _keys(g, n_pages, hkv, page, d)
    # an attention sink
    first = s["prefix_pages"][:1] if prefix else table[:, 0].clamp(min=0)
    k[first.long(), :, 0] *= 8.0
    s["k_cache"], s["k_scale"] = _quantise(k)
    s["v_cache"], s["v_scale"] = _quantise(_normal(g, n_pages, hkv, page, d))
    # the places behind a request's last token hold any bytes at all, codes and
    # scales that are no numbers among them
    last, end = (s["kv"].long() - 1) // page, s["kv"].long() % page
    tail = table.gather(1, last[:, None])[:, 0].long()
    behind = (torch.arange(page, device=DEVICE)[None, :] >= end[:, None]) & (end > 0)[:, None]
    for name in ("k", "v"):
        for part in ("_cache", "_scale"):
            x = s[name + part].view(torch.uint8)
            held = behind[:, None, :, None] if part == "_cache" else behind[:, None, :]
            x[tail] = x[tail].masked_fill(held, 255)
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = (torch.empty(hq, s["total"], dtype=torch.float32, device=DEVICE)
                if case["lse"] else None)
    if own:
        from paper_2507_21526_amd import binding
        s["plan"] = binding.PagedPlan(case["batch"], s["total"], hq, hkv, d, prefix=prefix > 0,
                                      ragged=s["cu_q"] is not None, q8=True)
    return s


# -------------------------------------------------------------- one pass
def run(state):
    s, case = state, state["case"]
    if own:
        return _run_own(s, case)
    return {"write": _plain_write, "read": _plain_read, "paged": _plain_paged}[case["op"]](s, case)


def _run_own(s, case):
    from paper_2507_21526_amd import binding
    if case["op"] == "write":
        binding.kv_cache_write(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"],
                               k_scale=s["k_scale"], v_scale=s["v_scale"])
        return {x: s[x] for x in ("k_cache", "k_scale", "v_cache", "v_scale")}
    if case["op"] == "read":
        binding.kv_cache_read(s["k_cache"], s["v_cache"], s["table"], s["cu"], s["k"], s["v"],
                              starts=s["starts"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return {"k": s["k"], "v": s["v"]}
    s["plan"].run(s["q"], s["k_cache"], s["v_cache"], s["o"], s["kv"], s["table"], cu_q=s["cu_q"],
                  prefix_pages=s["prefix_pages"], prefix_len=case["prefix"], lse=s["lse"],
                  softcap=case["softcap"] or None, slopes=s["slopes"], k_scale=s["k_scale"],
                  v_scale=s["v_scale"])
    return {"o": s["o"], "lse": s["lse"]}


def _plain_write(s, case):
    n, page = case["tokens"], case["page"]
    at = s["slots"][:n].long()

    def put(x, name):
        codes, scale = _quantise(x[:n])
        s[name + "_cache"].view(torch.uint8)[at // page, :, at % page] = codes.view(torch.uint8)
        s[name + "_scale"].view(torch.uint8)[at // page, :, at % page] = scale.view(torch.uint8)

    put(s["k"], "k")
    put(s["v"], "v")
    return {x: s[x] for x in ("k_cache", "k_scale", "v_cache", "v_scale")}


def _plain_read(s, case):
    n, page, cu = s["total"], case["page"], s["cu"].long()
    row = torch.arange(n, device=DEVICE)
    b = torch.searchsorted(cu[1:], row, right=True)
    pos = row - cu[b] + (s["starts"].long()[b] if s["starts"] is not None else 0)
    pages, place = s["table"][b, pos // page].long(), pos % page

    def get(name):
        if case["form"] == "bf16":
            s[name][:n] = s[name + "_cache"][pages, :, place]
            return
        scale = _scale(s[name + "_scale"].view(torch.uint8)[pages, :, place])[..., None]
        codes = s[name + "_cache"].view(torch.uint8)[pages, :, place]
        s[name][:n] = (codes.view(torch.float8_e4m3fn).float() * scale).bfloat16()

    get("k")
    get("v")
    return {"k": s["k"], "v": s["v"]}


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

    def values(name, at):
        scale = _scale(_taken(s[name + "_scale"], at))[..., None]
        return _taken(s[name + "_cache"], at).float() * scale

    def padded(name):
        x = values(name, pages).transpose(1, 2).reshape(batch, hkv, -1, d)[:, :, :keys]
        return torch.where(live[:, None, :, None], x, 0.0)

    pos = kv[:, None] - n_q[:, None] + t
    dist = (pos[:, :, None] - j).float()[:, None]  # [batch, 1, rows, keys]
    keep = (dist >= 0) & live[:, None, None]
    k, v = padded("k"), padded("v")
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(batch, hq, rows, keys)
    x = _scores(case, s["slopes"], x, dist)
    if prefix:  # the prefix's keys come before every request's own
        def shared(name):
            y = values(name, s["prefix_pages"].long()).transpose(0, 1)
            return y.reshape(hkv, -1, d)[:, :prefix]

        kp, vp = shared("k"), shared("v")
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


# ------------------------------------------------------------------- work
def _paged_work(case):
    kv, q = _paged_lens(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pairs = sum(b * (a + case["prefix"]) - b * (b - 1) // 2 for a, b in zip(kv, q))
    nbytes = 2 * hkv * (d + 1) * (sum(kv) + case["prefix"]) + 2 * 2 * sum(q) * hq * d
    nbytes += 4 * sum(_pages(n, case["page"]) for n in kv) + 8 * case["batch"]
    nbytes += 4 * hq * sum(q) if case["lse"] else 0
    return {"bytes": nbytes, "flops": 4 * d * hq * pairs}


def work(case):
    """Each input read and each output written once; two contractions per
    kept (row, key) pair."""
    hkv, d = case["hkv"], case["d"]
    if case["op"] == "write":
        n = case["tokens"]
        return {"bytes": 2 * n * hkv * (3 * d + 1) + 4 * (n + case["spare"]), "flops": 0}
    if case["op"] == "read":
        rows, skip = _read_lens(case)
        held = d + 1 if case["form"] == "8bit" else 2 * d
        entries = sum(_pages(a + b, case["page"]) - b // case["page"] for a, b in zip(rows, skip))
        return {"bytes": 2 * sum(rows) * hkv * (held + 2 * d) + 4 * entries + 8 * case["batch"],
                "flops": 0}
    return _paged_work(case)


# ------------------------------------------------------------ 64-bit form
def _nearest_e4m3(y):
    """The e4m3 value next to y (64 bits, at most 448), ties to the even one:
    steps of 1/8 of the power of two below |y|, and of 2^-9 under 2^-6."""
    _, e = torch.frexp(y)
    step = torch.exp2((e - 1).clamp(min=-6).to(torch.float64) - 3.0)
    return torch.round(y / step) * step


def _held64(x):
    """(elements, scales) that rows [..., d] are held as, in 64 bits."""
    x = x.to(torch.float64)
    top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    e = torch.full_like(top, float(LEAST_E))
    for n in range(LEAST_E, MOST_E):  # the least power of two that is enough
        e = torch.where(top > 448.0 * 2.0 ** n, torch.full_like(e, n + 1.0), e)
    scale = torch.exp2(e)
    most = torch.where(e == MOST_E, 240.0, 448.0)[..., None]
    y = _nearest_e4m3(x / scale[..., None])
    y = torch.minimum(torch.maximum(y, -most), most)
    return torch.where(torch.isfinite(x), y, torch.full_like(y, math.nan)), scale


def _values64(cache, scale):
    """What a cache holds, in 64 bits (bytes of scales that are no scale: NaN)."""
    if scale is None:
        return cache.to(torch.float64)
    b = scale.view(torch.uint8).to(torch.float64)
    two = torch.where(b == 255, torch.full_like(b, math.nan), torch.exp2(b - 127.0))
    return cache.float().to(torch.float64) * two[..., None]


def exact(case, seed):
    if case["op"] == "write":
        return _exact_write(case, seed)
    return _exact_read(case, seed) if case["op"] == "read" else _exact_paged(case, seed)


def _exact_write(case, seed):
    """Every head of every token to its place, a page's places laid out as
    one axis."""
    s = prepare(case, seed)
    at = s["slots"][:case["tokens"]].long()
    out = {}
    for name in ("k", "v"):
        pages, hkv, page, d = s[name + "_cache"].shape
        codes, scale = _held64(s[name][:case["tokens"]])
        flat = s[name + "_cache"].float().to(torch.float64).transpose(1, 2).reshape(-1, hkv, d)
        flat.index_copy_(0, at, codes)
        out[name + "_cache"] = flat.view(pages, page, hkv, d).transpose(1, 2).contiguous()
        flat = torch.exp2(s[name + "_scale"].view(torch.uint8).to(torch.float64) - 127.0)
        flat = flat.transpose(1, 2).reshape(-1, hkv)
        flat.index_copy_(0, at, scale)
        out[name + "_scale"] = flat.view(pages, page, hkv).transpose(1, 2).contiguous()
    return out


def _exact_read(case, seed):
    s = prepare(case, seed)
    rows, skip = _read_lens(case)
    out = {}
    for name in ("k", "v"):
        held = _values64(s[name + "_cache"], s[name + "_scale"])
        pages, hkv, page, d = held.shape
        held = held.transpose(1, 2)  # [pages, page, hkv, d]
        parts = []
        for b, (n, first) in enumerate(zip(rows, skip)):
            at = s["table"][b, first // page:_pages(first + n, page)].long()
            parts.append(held[at].reshape(-1, hkv, d)[first % page:first % page + n])
        parts.append(s[name][sum(rows):].to(torch.float64))
        out[name] = torch.cat(parts)
    return out


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


def _exact_paged(case, seed):
    if work(case)["flops"] > 3e12 or case["batch"] * case["hq"] > 20000:
        return None
    s = prepare(case, seed)
    hq, hkv, d, page, prefix = (case[x] for x in ("hq", "hkv", "d", "page", "prefix"))
    o = torch.zeros(s["total"], hq, d, dtype=torch.float64, device=DEVICE)
    lse = torch.full((hq, s["total"]), -math.inf, dtype=torch.float64, device=DEVICE)
    start = 0
    for b, (n, m) in enumerate(zip(s["kv_host"], s["q_host"])):
        mine = torch.arange(n, device=DEVICE)
        page_of, place = s["table"][b].long()[mine // page], mine % page
        if prefix:
            pre = torch.arange(prefix, device=DEVICE)
            page_of = torch.cat([s["prefix_pages"].long()[pre // page], page_of])
            place = torch.cat([pre % page, place])
        at = torch.arange(prefix + n, device=DEVICE)
        k = _values64(_taken(s["k_cache"], (page_of, slice(None), place)),
                      _taken(s["k_scale"], (page_of, slice(None), place)))
        v = _values64(_taken(s["v_cache"], (page_of, slice(None), place)),
                      _taken(s["v_scale"], (page_of, slice(None), place)))
        for r0 in range(0, m, 512):
            r1 = min(m, r0 + 512)
            row = prefix + n - m + torch.arange(r0, r1, device=DEVICE)
            dist = (row[:, None] - at).to(torch.float64)
            for h in range(hq):
                g = h // (hq // hkv)
                q = s["q"][start + r0:start + r1, h].to(torch.float64)
                a, e = _rows64(q, k[:, g], v[:, g], dist >= 0, dist, case,
                               None if s["slopes"] is None else s["slopes"][h].item())
                o[start + r0:start + r1, h], lse[h, start + r0:start + r1] = a, e
        start += m
    return {"o": o, "lse": lse if case["lse"] else None}
