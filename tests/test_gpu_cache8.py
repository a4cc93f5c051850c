"""GPU tests of the 8-bit cache: quantising writes, reads, and a serving step
over it.  Held values are compared exactly: scales and elements follow from the
row alone, and come back without rounding."""
import math

import pytest
import torch

from paper_2507_21526_amd import binding as B
from tests.cache8_ref import quantise, typed, values
from tests.serving_ref import attend, check, geometric_slopes

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _bytes(*shape, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, shape, generator=g, dtype=torch.uint8).cuda()


def _same(a, b):
    """Equal codes, any NaN for a NaN, and no sign asked of a zero."""
    x, y = a.view(torch.float8_e4m3fn).float(), b.view(torch.float8_e4m3fn).float()
    return bool(((x == y) | (x.isnan() & y.isnan())).all())


def _write(k, v, slots, pages, page, seed=0):
    """kv_cache_write of k, v into caches of random bytes; (before, after) as
    [k, k scales, v, v scales] bytes."""
    hkv, d = k.shape[1:]
    held = [_bytes(pages, hkv, page, d, seed=seed), _bytes(pages, hkv, page, seed=seed + 1),
            _bytes(pages, hkv, page, d, seed=seed + 2), _bytes(pages, hkv, page, seed=seed + 3)]
    before = [x.clone() for x in held]
    kc, ks = typed(*held[:2])
    vc, vs = typed(*held[2:])
    B.kv_cache_write(k, v, slots, kc, vc, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    return before, held


def _check_write(k, v, slots, pages, page, seed=0):
    before, held = _write(k, v, slots, pages, page, seed)
    for x, codes, scales, was, was_s in ((k, *held[:2], *before[:2]), (v, *held[2:], *before[2:])):
        want, want_s = was.clone(), was_s.clone()
        c, s = quantise(x)
        for t, at in enumerate(slots.tolist()):
            if 0 <= at < pages * page:
                want[at // page, :, at % page] = c[t].cuda()
                want_s[at // page, :, at % page] = s[t].cuda()
        assert torch.equal(scales, want_s)
        assert _same(codes, want)
        kept = torch.ones_like(was_s, dtype=torch.bool)
        for at in slots.tolist():
            if 0 <= at < pages * page:
                kept[at // page, :, at % page] = False
        assert torch.equal(codes[kept], was[kept])  # to the bit


@pytest.mark.parametrize("tokens,hkv,d,page,fused", [
    (1, 1, 64, 16, False), (1, 1, 128, 16, False), (7, 3, 128, 16, True), (333, 8, 128, 64, True),
    (64, 2, 64, 256, False), (500, 5, 64, 32, True), (17, 1, 128, 128, False)])
def test_write(tokens, hkv, d, page, fused):
    g = torch.Generator().manual_seed(tokens)
    size = torch.exp2(torch.randint(-12, 12, (tokens, 1, 1), generator=g).float())
    if fused:  # views of a projection's output, other strides for k and v
        x = (torch.randn(tokens, 2 * hkv + 3, d, generator=g) * size).bfloat16().cuda()
        k = x[:, 3:3 + hkv]
        v = torch.randn(hkv, tokens, d, generator=g).bfloat16().cuda().transpose(0, 1)
    else:
        k = (torch.randn(tokens, hkv, d, generator=g) * size).bfloat16().cuda()
        v = torch.randn(tokens, hkv, d, generator=g).bfloat16().cuda()
    pages = tokens // page + 4
    slots = torch.randperm(pages * page, generator=g)[:tokens].to(torch.int32)
    if tokens > 3:
        slots[1], slots[2], slots[3] = -1, pages * page, -2 ** 31  # skipped
    _check_write(k, v, slots.cuda(), pages, page, seed=tokens)


@pytest.mark.parametrize("d", [64, 128])
def test_write_of_every_value(d):
    """All bf16 bit patterns in rows of one size each (rows of 64 or 128 that
    follow one another), of mixed sizes, infinities and NaN among them; and
    each value beside one that sets the scale."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    rows = bits.reshape(-1, 1, d)
    mixed = bits[torch.randperm(65536, generator=torch.Generator().manual_seed(3))]
    mixed = mixed.reshape(-1, 1, d)
    fine = torch.where(torch.isfinite(mixed), mixed, 0.0)
    small = torch.where(fine.abs() < 2.0 ** 10, fine, 1.0)
    small[:, 0, 5] = 1000.0
    for x in (rows, mixed, fine, small):
        n = x.shape[0]
        _check_write(x.cuda(), x.flip(0).cuda(), torch.arange(n, dtype=torch.int32).cuda(),
                     n // 16, 16)


def test_write_of_rows_at_a_scale_s_border():
    """The largest value of a row at, just under and just over 448 2^e, at the
    ends of the scales, and ties between elements."""
    rows = []
    for e in (-140, -110, -101, -100, -99, -5, 0, 7, 100, 118, 119):
        for m in (1.0, 1.5, 1.7421875, 1.75, 1.7578125, 1.9921875):
            rows.append([m * 2.0 ** (e + 8)] + [m * 2.0 ** (e + 8 - i) for i in range(63)])
    for e in range(-9, 9):  # halves of steps: 1 + i / 16
        rows.append([256.0] + [(1 + (i % 16) / 16) * 2.0 ** (e - i // 16) for i in range(63)])
    x = torch.tensor(rows, dtype=torch.float64).float().bfloat16()[:, None]
    x[::3] *= -1
    n = x.shape[0]
    _check_write(x.cuda(), x.flip(0).cuda(), torch.arange(n, dtype=torch.int32).cuda(), n // 16 + 1,
                 16)


def test_write_of_more_rows_than_threads():
    """2^28 rows and more: one row's views repeated, a few of them with a slot."""
    n, hkv, d = (1 << 25) + 5, 8, 128
    k = torch.randn(1, hkv, d, device="cuda").bfloat16()
    v = torch.randn(1, hkv, d, device="cuda").bfloat16()
    held = [torch.zeros(2, hkv, 16, d, dtype=torch.uint8, device="cuda"),
            torch.zeros(2, hkv, 16, dtype=torch.uint8, device="cuda")]
    held += [x.clone() for x in held]
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 1, 1 << 24, n - 6, n - 1], device="cuda")
    slots[at] = torch.arange(3, 8, dtype=torch.int32, device="cuda")
    kc, ks = typed(*held[:2])
    vc, vs = typed(*held[2:])
    B.kv_cache_write(k.expand(n, hkv, d), v.expand(n, hkv, d), slots, kc, vc, k_scale=ks,
                     v_scale=vs)
    for x, codes, scales in ((k, *held[:2]), (v, *held[2:])):
        c, s = quantise(x[0])
        assert _same(codes[0, :, 3:8], c.cuda()[:, None].expand(hkv, 5, d))
        assert torch.equal(scales[0, :, 3:8], s.cuda()[:, None].expand(hkv, 5))
        for y in (codes, scales):
            assert not bool(y[0, :, :3].any()) and not bool(y[0, :, 8:].any())
            assert not bool(y[1].any())


@pytest.mark.parametrize("d", [64, 128])
def test_read_of_every_code_and_scale(d):
    """256 codes under 256 scale bytes come back as what they stand for,
    rounded to bf16 where a foreign scale leaves its range."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(d // 64).reshape(-1, d)  # [4, d]
    k8 = codes.repeat(256, 1).reshape(4, 256, 1, d).transpose(0, 1).reshape(1024, d)
    s = torch.arange(256, dtype=torch.uint8).repeat_interleave(4)
    k8, v8 = k8.reshape(64, 1, 16, d).cuda(), k8.flip(0).contiguous().reshape(64, 1, 16, d).cuda()
    ks, vs = s.reshape(64, 1, 16).cuda(), s.flip(0).contiguous().reshape(64, 1, 16).cuda()
    k = torch.zeros(1024, 1, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    kc, kt = typed(k8, ks)
    vc, vt = typed(v8, vs)
    B.kv_cache_read(kc, vc, torch.arange(64, dtype=torch.int32, device="cuda")[None],
                    _ints([0, 1024]), k, v, k_scale=kt, v_scale=vt)
    for got, c, x in ((k, k8, ks), (v, v8, vs)):
        want = values(c, x).bfloat16().reshape(1024, 1, d)
        assert bool(((got == want) | (got.isnan() & want.isnan())).all())


def _cache(pages, hkv, page, d, q8, seed):
    """(k, v, {scales}, held k, held v in bf16)."""
    g = torch.Generator().manual_seed(seed)
    x = [torch.randn(pages, hkv, page, d, generator=g).bfloat16() for _ in range(2)]
    if not q8:
        return x[0].cuda(), x[1].cuda(), {}, x[0].cuda(), x[1].cuda()
    (k, ks), (v, vs) = quantise(x[0]), quantise(x[1])
    held = [values(k, ks).bfloat16().cuda(), values(v, vs).bfloat16().cuda()]
    k, ks = typed(k.cuda(), ks.cuda())
    v, vs = typed(v.cuda(), vs.cuda())
    return k, v, dict(k_scale=ks, v_scale=vs), *held


def _want_rows(held, table, cu, starts, page, out):
    """out with the rows of kv_cache_read in place."""
    out = out.clone()
    for b in range(len(cu) - 1):
        for r in range(cu[b], cu[b + 1]):
            pos = starts[b] + r - cu[b]
            at = table[b][pos // page] if 0 <= pos and pos // page < len(table[b]) else -1
            out[r] = held[at, :, pos % page] if 0 <= at < held.shape[0] else math.nan
    return out


READS = [
    # rows read, positions skipped, hkv, d, page, spare rows
    ([1], [0], 1, 64, 16, 0),
    ([1], [15], 1, 128, 16, 3),
    ([15, 16, 17, 0, 1], [0, 1, 16, 5, 31], 3, 128, 16, 2),
    ([0, 0, 40], [0, 7, 100], 8, 64, 32, 0),
    ([300, 513], [0, 0], 2, 128, 256, 40),
    ([70, 1, 33], [64, 63, 1], 5, 64, 64, 1),
    ([130], [200], 2, 64, 128, 0),
]


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("case", READS, ids=lambda c: f"{max(c[0])}-{max(c[1])}-{c[2]}-{c[3]}-"
                         f"{c[4]}")
@pytest.mark.parametrize("layout", ["plain", "heads", "halves", "turned"])
def test_read(case, q8, layout):
    rows, skip, hkv, d, page, spare = case
    cu = [0]
    for n in rows:
        cu.append(cu[-1] + n)
    need = [-(-(n + s) // page) for n, s in zip(rows, skip)]
    pages, width = sum(need) + 3, max(need) + 1
    kc, vc, scales, hk, hv = _cache(pages, hkv, page, d, q8, sum(rows))
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).tolist()
    table = [[ids.pop() for _ in range(n)] + [-1] * (width - n) for n in need]
    total = cu[-1] + spare
    if layout == "plain":
        k, v = (torch.full((total, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
                for _ in range(2))
    elif layout == "heads":  # a fused buffer [T, 2 heads + 1, d]
        buf = torch.full((total, 2 * hkv + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
        k, v = buf[:, :hkv], buf[:, hkv + 1:]
    elif layout == "halves":  # K and V of a head side by side
        buf = torch.full((total, hkv, 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
        k, v = buf[:, :, 0], buf[:, :, 1]
    else:  # heads outermost
        buf = torch.full((hkv, 2, total, d), 7.0, dtype=torch.bfloat16, device="cuda")
        k, v = buf[:, 0].transpose(0, 1), buf[:, 1].transpose(0, 1)
    wk = _want_rows(hk, table, cu, skip, page, k)
    wv = _want_rows(hv, table, cu, skip, page, v)
    starts = None if not any(skip) else _ints(skip)
    B.kv_cache_read(kc, vc, _ints(table), _ints(cu), k, v, starts=starts, **scales)
    torch.cuda.synchronize()
    assert torch.equal(k, wk) and torch.equal(v, wv)
    if layout == "heads":
        assert bool((buf[:, hkv] == 7.0).all())


@pytest.mark.parametrize("q8", [False, True])
def test_read_of_rows_that_no_page_holds(q8):
    page, hkv, d = 16, 2, 64
    kc, vc, scales, hk, hv = _cache(6, hkv, page, d, q8, 4)
    cu, starts = [0, 40, 60, 61, 70], [-3, 40, 2 ** 31 - 1, -2 ** 31]
    table = [[1, 6, 2], [0, 3, -1], [4, 4, 4], [5, 2 ** 31 - 1, -2 ** 31]]
    out = torch.full((73, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    k, v = out.clone(), out.clone()
    B.kv_cache_read(kc, vc, _ints(table), _ints(cu), k, v, starts=_ints(starts), **scales)
    for got, held in ((k, hk), (v, hv)):
        want = _want_rows(held, table, cu, starts, page, out)
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(), want.nan_to_num())
        assert bool(got[:3].isnan().all()) and bool(got[3:19].isfinite().all())
        assert bool(got[60:70].isnan().all()) and bool((got[70:] == 7.0).all())
    for bad in ([0, 20, 10, 30, 40], [1, 2, 3, 4, 5], [0, 1, 2, 3, 74], [0, -1, 2, 3, 4],
                [0, 0, 0, 0, -1]):
        k, v = out.clone(), out.clone()
        B.kv_cache_read(kc, vc, _ints(table), _ints(bad), k, v, **scales)
        assert bool(k.isnan().all()) and bool(v.isnan().all()), bad


@pytest.mark.parametrize("q8", [False, True])
def test_read_of_the_largest_batch(q8):
    page, hkv, d, b = 16, 1, 64, 1024
    kc, vc, scales, hk, hv = _cache(50, hkv, page, d, q8, 5)
    cu, starts = [0], []
    for i in range(b):
        cu.append(cu[-1] + i % 4)
        starts.append(i % 29)
    table = [[(7 * i) % 50, (11 * i + 3) % 50] for i in range(b)]
    k = torch.zeros(cu[-1], hkv, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    B.kv_cache_read(kc, vc, _ints(table), _ints(cu), k, v, starts=_ints(starts), **scales)
    pos = [(b, starts[b] + i) for b in range(1024) for i in range(cu[b + 1] - cu[b])]
    at = torch.tensor([table[i][p // page] if p // page < 2 else -1 for i, p in pos]).cuda()
    place = torch.tensor([p % page for _, p in pos]).cuda()
    assert torch.equal(k, hk[at, :, place]) and torch.equal(v, hv[at, :, place])


def test_read_without_requests_or_pages():
    k = torch.full((3, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    kc, vc, scales, _, _ = _cache(1, 2, 16, 64, True, 6)
    B.kv_cache_read(kc, vc, _ints([]).reshape(0, 4), _ints([0]), k, v, **scales)
    assert bool((k == 7.0).all())
    none = kc[:0], vc[:0], {n: x[:0] for n, x in scales.items()}
    B.kv_cache_read(*none[:2], _ints([[0]]), _ints([0, 2]), k, v, **none[2])
    assert bool(k[:2].isnan().all()) and bool((k[2] == 7.0).all())
    B.kv_cache_read(kc, vc, _ints([[], []]).reshape(2, 0), _ints([0, 2, 3]), k, v, **scales)
    assert bool(k.isnan().all())


def test_read_past_32_bits():
    """Pages whose byte offset in the cache passes 2^32."""
    page, hkv, d, pages = 256, 8, 128, 17000  # 17000 * 8 * 256 * 128 = 4.5e9
    kc, vc = (torch.zeros(pages, hkv, page, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(pages, hkv, page, dtype=torch.uint8, device="cuda") for _ in range(2))
    x = torch.randn(5, hkv, d, generator=torch.Generator().manual_seed(8)).bfloat16().cuda()
    slots = [16999 * 256 + 255, 16400 * 256, -1, 3 * 256 + 17, 16999 * 256 + 254]
    kt, kst = typed(kc, ks)
    vt, vst = typed(vc, vs)
    B.kv_cache_write(x, -x, _ints(slots), kt, vt, k_scale=kst, v_scale=vst)
    c, s = quantise(x)
    want = values(c, s).bfloat16().cuda()
    k = torch.zeros(4, hkv, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    B.kv_cache_read(kt, vt, _ints([[16999], [16400], [3]]), _ints([0, 2, 3, 4]), k, v,
                    starts=_ints([254, 0, 17]), k_scale=kst, v_scale=vst)
    assert torch.equal(k, want[[4, 0, 1, 3]]) and torch.equal(v, -want[[4, 0, 1, 3]])


def test_read_of_more_rows_than_workgroups():
    """2^26 rows and more: workgroups take several blocks of rows."""
    n, page = (1 << 26) + 37, 256
    kc, vc, scales, hk, hv = _cache(8, 1, page, 64, True, 11)
    table = torch.randint(0, 8, (1, -(-n // page)), dtype=torch.int32, device="cuda")
    k = torch.zeros(n + 2, 1, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    B.kv_cache_read(kc, vc, table, _ints([0, n]), k, v, **scales)
    for first in (0, 1 << 25, (1 << 26) - 70000, n - 70000):
        row = torch.arange(first, first + 70000, device="cuda")
        at = table[0, row // page].long()
        assert torch.equal(k[row], hk[at, :, row % page])
        assert torch.equal(v[row], hv[at, :, row % page])
    assert not bool(k[n:].any()) and not bool(v[n:].any())


def test_write_and_read_on_another_stream_and_captured():
    """Both calls captured in one graph, replayed with other rows and offsets
    between eager work; and on a stream of their own."""
    page, hkv, d, pages = 16, 2, 128, 8
    held = [torch.zeros(pages, hkv, page, d, dtype=torch.uint8, device="cuda"),
            torch.zeros(pages, hkv, page, dtype=torch.uint8, device="cuda")]
    held += [x.clone() for x in held]
    kc, ks = typed(*held[:2])
    vc, vs = typed(*held[2:])
    x = torch.zeros(9, 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
    slots, table, cu = _ints([0] * 9), _ints([[0, 0], [0, 0]]), _ints([0, 0, 0])
    k, v = (torch.zeros(9, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step(stream=None):
        B.kv_cache_write(x[:, :hkv], x[:, hkv:], slots, kc, vc, k_scale=ks, v_scale=vs,
                         stream=stream)
        B.kv_cache_read(kc, vc, table, cu, k, v, k_scale=ks, v_scale=vs, stream=stream)

    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(9)
    for i in range(6):
        x.copy_(torch.randn(9, 2 * hkv, d, generator=g) * 2.0 ** (4 * i))
        a, b = (2 * i) % 8, (2 * i + 3) % 8
        n = 1 + i
        slots.copy_(torch.tensor([a * 16 + j for j in range(n)] +
                                 [b * 16 + j for j in range(9 - n)], dtype=torch.int32))
        table.copy_(torch.tensor([[a, -1], [b, -1]], dtype=torch.int32))
        cu.copy_(torch.tensor([0, n, 9], dtype=torch.int32))
        k.fill_(7.0)
        torch.cuda.synchronize()
        if i % 2:
            graph.replay()
        else:
            step(side)
        torch.cuda.synchronize()
        for got, rows in ((k, x[:, :hkv]), (v, x[:, hkv:])):
            c, s = quantise(rows)
            assert torch.equal(got.cpu(), values(c, s).bfloat16()), i
        torch.zeros(1000, device="cuda").add_(1)


@pytest.mark.parametrize("score", ["plain", "both"])
def test_a_serving_run(score):
    """Prompts into the 8-bit cache and back, through the prefill pass, then
    decoded tokens through a captured step of map, write and attention: every row
    is that of attention over the held values."""
    hq, hkv, d, page, steps = 8, 2, 128, 16, 4
    lens = [130, 17, 64]
    b, width = 3, 12
    cap, sl = (25.0, geometric_slopes(hq)) if score == "both" else (None, None)
    g = torch.Generator().manual_seed(50)
    seqs = [[torch.randn(n + steps, h, d, generator=g).bfloat16().cuda() for h in (hq, hkv, hkv)]
            for n in lens]
    held = [[values(*quantise(s[i])).bfloat16().cuda() for i in (1, 2)] for s in seqs]
    cu = [0, 130, 147, 211]
    q, k, v = (torch.cat([s[i][:n] for s, n in zip(seqs, lens)]) for i in range(3))
    store = [torch.full((40, hkv, page, d), 255, dtype=torch.uint8, device="cuda"),
             torch.full((40, hkv, page), 255, dtype=torch.uint8, device="cuda")]
    store += [x.clone() for x in store]
    kc, ks = typed(*store[:2])
    vc, vs = typed(*store[2:])
    scales = dict(k_scale=ks, v_scale=vs)
    table = torch.full((b, width), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.randperm(40, device="cuda").to(torch.int32), _ints([40])
    cached, kv, cu_new = _ints([0, 0, 0]), _ints([0] * 3), _ints([0] * 4)
    slots, state = _ints([0] * 211), _ints([0, 0])
    B.page_map(cached, _ints(lens), table, free, n_free, page, kv, cu_new, slots, state)
    B.kv_cache_write(k, v, slots, kc, vc, **scales)
    # the prompts' held keys and values back, and the dense pass over them
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    B.kv_cache_read(kc, vc, table, cu_new, rk, rv, **scales)
    for i, n in enumerate(lens):
        assert torch.equal(rk[cu[i]:cu[i + 1]], held[i][0][:n])
        assert torch.equal(rv[cu[i]:cu[i + 1]], held[i][1][:n])
    o = torch.empty_like(q)
    B.Plan("causal", cu, 0, 1, 0, 64, hq, d).run(q, rk, rv, o, softcap=cap, slopes=sl)
    for i, n in enumerate(lens):
        dist = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
        ref = attend(seqs[i][0][:n], held[i][0][:n], held[i][1][:n], dist >= 0, dist, d ** -0.5,
                     cap, sl)
        check(o[cu[i]:cu[i + 1]], None, ref, torch.bfloat16, f"prompt {i}")
    # the same rows as a piece over the cache
    piece = torch.empty_like(q)
    B.PagedPlan(b, 211, hq, hkv, d, ragged=True, q8=True).run(
        q, kc, vc, piece, kv, table, cu_q=cu_new, softcap=cap, slopes=sl, **scales)
    for i, n in enumerate(lens):
        dist = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
        ref = attend(seqs[i][0][:n], held[i][0][:n], held[i][1][:n], dist >= 0, dist, d ** -0.5,
                     cap, sl)
        check(piece[cu[i]:cu[i + 1]], None, ref, torch.bfloat16, f"piece {i}")
    # one decode step, captured
    one, nk = _ints([1, 1, 1]), torch.zeros(b, hkv, d, dtype=torch.bfloat16, device="cuda")
    nq, nv = torch.zeros(b, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(nk)
    no, nlse = torch.zeros_like(nq), torch.zeros(hq, b, device="cuda")
    slot1 = _ints([0] * 3)
    plan = B.PagedPlan(b, b, hq, hkv, d, q8=True)

    def step():
        cached.copy_(kv)
        n_free.copy_(state[:1])
        B.page_map(cached, one, table, free, n_free, page, kv, cu_new, slot1, state)
        B.kv_cache_write(nk, nv, slot1, kc, vc, **scales)
        plan.run(nq, kc, vc, no, kv, table, lse=nlse, softcap=cap, slopes=sl, **scales)

    graph = None
    for t in range(steps):
        for i in range(b):
            nq[i], nk[i], nv[i] = (s[lens[i] + t] for s in seqs[i])
        if t == 0:
            step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert state[1] == 0 and kv.tolist() == [n + t + 1 for n in lens]
        for i, n in enumerate(lens):
            m = n + t + 1
            dist = (m - 1 - torch.arange(m, device="cuda"))[None]
            ref = attend(seqs[i][0][m - 1:m], held[i][0][:m], held[i][1][:m], dist >= 0, dist,
                         d ** -0.5, cap, sl)
            check(no[i:i + 1], nlse.t()[i:i + 1], ref, torch.bfloat16, f"step {t} request {i}")
