"""GPU tests of attention over the 8-bit paged cache, against 64 bits over the
held values."""
import math
import random

import pytest
import torch

from paper_2507_21526_amd import binding as B
from tests.cache8_ref import Cache8
from tests.serving_ref import attend, check, geometric_slopes

pytestmark = pytest.mark.gpu


def _call(c, q, q_lens, dtype=torch.bfloat16, softcap=None, slopes=None, lse=True, ragged=None,
          behind=0, plan=None):
    """One call; `behind` rows after the last request.  (o, lse [R, hq])."""
    total, hq, d = q.shape
    ragged = any(n != 1 for n in q_lens) if ragged is None else ragged
    cu = [0]
    for n in q_lens:
        cu.append(cu[-1] + n)
    assert cu[-1] + behind == total
    cu = torch.tensor(cu, dtype=torch.int32, device=q.device) if ragged else None
    k, v, scales = c.tensors()
    plan = plan or B.PagedPlan(len(q_lens), total, hq, k.shape[1], d, prefix=c.prefix > 0,
                               ragged=ragged, q8=True)
    plan.workspace.fill_(0xff)  # NaN bit patterns
    o = torch.full(q.shape, 7.0, dtype=dtype, device=q.device)
    l = torch.full((hq, total), 7.0, device=q.device) if lse else None
    plan.run(q, k, v, o, c.kv_lens, c.table, cu_q=cu,
             prefix_pages=c.prefix_pages if c.prefix else None, prefix_len=c.prefix, lse=l,
             softcap=softcap, slopes=slopes, **scales)
    torch.cuda.synchronize()
    if behind:
        assert bool((o[-behind:] == 7.0).all()), "rows behind the last request"
        assert not lse or bool((l[:, -behind:] == 7.0).all())
        o = o[:-behind]
        l = l[:, :-behind] if lse else None
    return o, l.t() if lse else None


def _q(total, hq, d, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(total, hq, d, generator=g).bfloat16().cuda()


SINGLE = [
    # own lengths, hq, hkv, d, page, prefix
    ([1], 1, 1, 64, 16, 0),
    ([1, 15, 16, 17, 31, 32, 33, 127, 128, 129], 4, 1, 128, 16, 0),
    ([0, 5, 0, 0, 900, 0], 8, 2, 64, 32, 0),             # requests without keys
    ([700, 3, 64], 7, 1, 128, 64, 0),
    ([513, 1000, 2, 77], 16, 2, 128, 128, 0),            # eight heads to a kv head
    ([300, 301, 255, 256, 257], 10, 2, 64, 256, 0),
    ([20011], 3, 1, 128, 16, 0),                         # one request over the whole chip
    ([9001, 4, 12007], 8, 8, 64, 32, 0),                 # one head to a kv head
    ([1 + 37 * (i % 11) for i in range(300)], 6, 1, 64, 16, 0),  # many short ones
    ([10, 200, 1, 513], 4, 1, 128, 16, 1),               # a prefix of one key
    ([10, 200, 1, 0], 4, 1, 64, 16, 37),                 # 16 rows: all fit one row tile
    ([10, 200, 1, 700, 33, 8, 90, 64, 65], 16, 4, 128, 64, 1000),
    ([5 + i for i in range(70)], 8, 2, 64, 32, 4133),
    ([3, 0, 2], 8, 8, 128, 16, 300),
    ([40000, 100], 5, 1, 128, 256, 0),
]


@pytest.mark.parametrize("case", SINGLE, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}-{c[2]}-"
                         f"{c[3]}-{c[4]}-{c[5]}")
@pytest.mark.parametrize("score", ["plain", "cap", "slopes", "both"])
def test_single_tokens(case, score):
    lens, hq, hkv, d, page, prefix = case
    c = Cache8(lens, hkv, d, page, prefix, seed=len(lens) + hq)
    q = _q(len(lens), hq, d, 5)
    cap = 12.0 if score in ("cap", "both") else None
    sl = geometric_slopes(hq) if score in ("slopes", "both") else None
    dtype = torch.float32 if score in ("plain", "both") else torch.bfloat16
    o, l = _call(c, q, [1] * len(lens), dtype, cap, sl)
    check(o, l, c.reference(q, [1] * len(lens), d ** -0.5, cap, sl), dtype, f"{case} {score}")


RAGGED = [
    # own lengths, query lengths, hq, hkv, d, page, prefix, rows behind
    ([9, 300, 40, 7], [1, 5, 0, 3], 4, 1, 64, 16, 0, 2),
    ([9, 300, 40, 7], [1, 4, 2, 7], 8, 2, 128, 32, 0, 0),     # drafted tokens
    ([2, 0, 33], [5, 2, 33], 4, 2, 64, 16, 0, 0),             # rows before the first key
    ([257], [257], 4, 1, 128, 16, 0, 1),                      # a whole prompt
    ([1000, 130, 64, 5], [300, 129, 1, 5], 8, 1, 64, 64, 0, 0),
    ([2500, 70], [600, 70], 10, 2, 128, 128, 0, 3),
    ([700, 41, 1], [90, 41, 1], 7, 1, 64, 16, 129, 0),
    ([12, 30, 5, 4], [2, 3, 1, 6], 8, 2, 128, 16, 77, 1),     # prefix, rows before the first key
    ([40] * 20, [3] * 20, 6, 2, 64, 32, 515, 0),
    ([3000], [1], 4, 1, 128, 16, 0, 0),                       # one row given as ragged
    ([300, 20], [250, 20], 8, 1, 128, 256, 1000, 0),          # pieces behind a prefix
]


@pytest.mark.parametrize("case", RAGGED, ids=lambda c: f"{max(c[0])}-{max(c[1])}-{c[2]}-{c[3]}-"
                         f"{c[4]}-{c[5]}-{c[6]}")
@pytest.mark.parametrize("score", ["plain", "cap", "slopes", "both"])
def test_several_tokens(case, score):
    lens, ql, hq, hkv, d, page, prefix, behind = case
    c = Cache8(lens, hkv, d, page, prefix, seed=hq)
    q = _q(sum(ql) + behind, hq, d, 6)
    cap = 20.0 if score in ("cap", "both") else None
    sl = geometric_slopes(hq) if score in ("slopes", "both") else None
    dtype = torch.bfloat16 if score in ("cap", "both") else torch.float32
    o, l = _call(c, q, ql, dtype, cap, sl, ragged=True, behind=behind)
    check(o, l, c.reference(q, ql, d ** -0.5, cap, sl), dtype, f"{case} {score}")


def test_against_the_bf16_cache():
    """The same values held in either form: the results differ by what rounding
    a probability before or after its value's scale does, nothing (a power of
    two), and by the order of sums."""
    for lens, ql, prefix, d in (([700, 33, 1], [1, 1, 1], 0, 128), ([700, 90], [200, 90], 100, 64),
                                ([90, 70], [4, 3], 300, 128)):
        c = Cache8(lens, 2, d, 16, prefix, seed=31)
        q = _q(sum(ql), 8, d, 31)
        o, l = _call(c, q, ql, torch.float32, ragged=True)
        o16, l16 = torch.empty_like(o), torch.empty(8, sum(ql), device="cuda")
        cu = torch.tensor([0, *torch.tensor(ql).cumsum(0).tolist()], dtype=torch.int32).cuda()
        B.PagedPlan(len(ql), sum(ql), 8, 2, d, prefix=prefix > 0, ragged=True).run(
            q, c.k, c.v, o16, c.kv_lens, c.table, cu_q=cu,
            prefix_pages=c.prefix_pages if prefix else None, prefix_len=prefix, lse=l16)
        ref = c.reference(q, ql, d ** -0.5)
        check(o, l, ref, torch.float32, f"8 bits {d}")
        check(o16, l16.t(), ref, torch.float32, f"16 bits {d}")


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_batch(d, ragged):
    lens = [(7 * i) % 90 for i in range(1024)]
    ql = [(i % 3) for i in range(1024)] if ragged else [1] * 1024
    c = Cache8(lens, 1, d, 16, prefix=20, seed=8)
    q = _q(sum(ql), 2, d, 9)
    o, l = _call(c, q, ql, torch.float32)
    starts = [0]
    for n in ql:
        starts.append(starts[-1] + n)
    some = [i for i in list(range(0, 1024, 37)) + [1023] if ql[i]]
    at = torch.cat([torch.arange(starts[i], starts[i + 1]) for i in some]).cuda()
    c.lens, c.table = [lens[i] for i in some], c.table[some]
    check(o[at], l[at], c.reference(q[at], [ql[i] for i in some], d ** -0.5), torch.float32,
          "1024 requests")


def test_many_row_tiles():
    """Near the limit of row tiles: a long piece of a prompt, many heads."""
    c = Cache8([30000, 40], 1, 64, 256, seed=9)
    q = _q(30000 + 2, 8, 64, 10)
    o, l = _call(c, q, [30000, 2], ragged=True)
    rows = torch.cat([torch.arange(0, 30000, 1777), torch.tensor([29999])]).cuda()
    k, v = c.keys(0)
    dist = rows[:, None] - torch.arange(30000, device="cuda")
    check(o[rows], l[rows], attend(q[rows], k, v, dist >= 0, dist, 0.125), torch.bfloat16, "piece")
    c.lens, c.table = [40], c.table[1:]
    check(o[30000:], l[30000:], c.reference(q[30000:], [2], 0.125), torch.bfloat16, "two rows")


@pytest.mark.parametrize("bad", ["element", "scale", "large"])
@pytest.mark.parametrize("d,ql", [(64, 4), (128, 4), (128, 50), (64, 50)])
def test_values_behind_a_row(bad, d, ql):
    """A NaN value, element or scale, reaches the rows that keep its key, and
    no other; a value of 2^127 (448 2^118 there) stays finite in them."""
    lens = [150, 60]
    c = Cache8(lens, 1, d, 16, seed=1)
    q = _q(2 * ql, 4, d, 8)
    for b, back in ((0, 2), (1, 1)):  # the last but one key, the last key
        p = lens[b] - back
        page = int(c.table[b, p // 16])
        if bad == "element":
            c.put("v", page, p % 16, code=127, at=3)
            c.put("v", page, p % 16, code=255, at=d - 1)
        elif bad == "scale":
            c.put("v", page, p % 16, scale=255)
        else:
            c.put("v", page, p % 16, scale=127 + 100)
    o, l = _call(c, q, [ql, ql], torch.float32, ragged=True)
    ref = c.reference(q, [ql, ql], d ** -0.5)
    keeps = ~torch.isfinite(ref[0]).all(-1).all(-1)
    # two rows of the first request, one of the second
    assert int(keeps.sum()) == (0 if bad == "large" else 3)
    check(o, l, ref, torch.float32, f"{bad} d {d} rows {ql}")


@pytest.mark.parametrize("part", ["element", "scale"])
@pytest.mark.parametrize("d,ql", [(64, 3), (128, 3), (128, 50), (64, 50)])
def test_keys_that_are_nan(part, d, ql):
    """A NaN key makes the rows that keep it NaN, and no earlier row."""
    n = 100
    c = Cache8([n, 40], 1, d, 16, seed=2)
    q = _q(ql + 1, 4, d, 8)
    p = n - 2
    page = int(c.table[0, p // 16])
    if part == "element":
        c.put("k", page, p % 16, code=127, at=d - 2)
    else:
        c.put("k", page, p % 16, scale=255)
    o, l = _call(c, q, [ql, 1], torch.float32, ragged=True)
    ref = c.reference(q, [ql, 1], d ** -0.5)
    assert bool(o[ql - 2:ql].isnan().all()) and bool(l[ql - 2:ql].isnan().all())
    rest = torch.cat([torch.arange(ql - 2), torch.tensor([ql])]).cuda()
    check(o[rest], l[rest], tuple(x[rest] for x in ref), torch.float32, f"{part} {d} {ql}")


@pytest.mark.parametrize("hq,d", [(1, 128), (1, 64), (3, 128), (8, 64)])
def test_values_in_every_part_of_a_step(hq, d):
    """Rows of one head or few: at one step some waves of a row tile drop keys
    and others keep all of them.  A value of each key in turn is NaN; no row
    before the key sees it."""
    n = 128
    c = Cache8([n], 1, d, 16, seed=5)
    q = _q(n, hq, d, 12)
    clean, _ = _call(c, q, [n], torch.float32, ragged=True)
    keep = c.v8.clone(), c.vs.clone()
    for j in range(0, n, 3):
        c.v8.copy_(keep[0])
        c.vs.copy_(keep[1])
        page, place = int(c.table[0, j // 16]), j % 16
        if j % 2:
            c.vs[page, 0, place] = 255
        else:
            c.v8[page, 0, place, j % d] = 127
        o, _ = _call(c, q, [n], torch.float32, ragged=True)
        assert bool(torch.isfinite(o[:j]).all()), j
        # the same sums, key by key: bits may differ by their order
        assert float((o[:j] - clean[:j]).abs().max() if j else 0.0) < 1e-5, j
        assert not bool(torch.isfinite(o[j:, :, j % d]).any()), j


@pytest.mark.parametrize("d,ql", [(64, 1), (128, 1), (128, 60), (64, 60)])
def test_foreign_scales(d, ql):
    """Scale bytes that the write does not make: 0 and 1, up to 200."""
    c = Cache8([200], 1, d, 16, seed=6)
    q = _q(ql, 4, d, 13)
    for p, (ks, vs) in enumerate([(0, 0), (1, 1), (9, 20), (26, 200), (127, 0), (0, 190)]):
        page = int(c.table[0, p // 16])
        c.put("k", page, p % 16, scale=ks)
        c.put("v", page, p % 16, scale=vs)
    o, l = _call(c, q, [ql], torch.float32, ragged=ql > 1)
    check(o, l, c.reference(q, [ql], d ** -0.5), torch.float32, f"foreign {d} {ql}")


@pytest.mark.parametrize("d,ql", [(64, 1), (128, 1), (128, 60), (64, 60)])
@pytest.mark.parametrize("e", [-100, -60, 60])
def test_values_of_any_size(d, ql, e):
    """Values whose sizes lie far from 1, all scales alike: the result scales
    with them (2^e, so exactly)."""
    c = Cache8([300], 2, d, 16, seed=7)
    q = _q(ql, 8, d, 14)
    c.vs.fill_(127)
    c.v = (c.v8.view(torch.float8_e4m3fn).float()).bfloat16()
    o, l = _call(c, q, [ql], torch.float32, ragged=ql > 1)
    ref = c.reference(q, [ql], d ** -0.5)
    check(o, l, ref, torch.float32, f"size 0 {d} {ql}")
    c.vs.fill_(127 + e)
    o2, l2 = _call(c, q, [ql], torch.float32, ragged=ql > 1)
    assert torch.equal(l, l2)
    # bf16 weights below 2^-126 may be lost: at most 2^-26 of the row's largest
    # (for e = -100), each times 448
    size = ref[2].abs().max() * 2.0 ** -14
    assert float((o2.double() * 2.0 ** -e - o.double()).abs().max()) <= float(size)
    if e != -100:
        assert torch.equal(o2, torch.ldexp(o, torch.tensor(e, device="cuda")))


def test_bad_pages_and_lengths_show():
    """A page id outside the cache, and a length past the table, give NaN in
    the rows of that request and nowhere else; bad query offsets in all."""
    lens = [100, 90, 80]
    c = Cache8(lens, 2, 64, 16, seed=2)
    q = _q(3, 4, 64, 9)
    good, gl = _call(c, q, [1, 1, 1], torch.float32)
    keep_table, keep_lens = c.table.clone(), c.kv_lens.clone()
    for page in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.table[1, 3] = page
        o, l = _call(c, q, [1, 1, 1], torch.float32)
        assert bool(torch.isnan(o[1]).all()) and bool(torch.isnan(l[1]).all())
        assert torch.equal(o[[0, 2]], good[[0, 2]]) and torch.equal(l[[0, 2]], gl[[0, 2]])
        c.table.copy_(keep_table)
    # an entry behind the last key is not read
    c.table[1, 6] = -5
    o, _ = _call(c, q, [1, 1, 1], torch.float32)
    assert torch.equal(o, good)
    for n in (c.table.shape[1] * 16 + 1, 2 ** 31 - 1):
        c.kv_lens[2] = n
        o, l = _call(c, q, [1, 1, 1], torch.float32)
        assert bool(torch.isnan(o[2]).all()) and bool(torch.isnan(l[2]).all())
        assert torch.equal(o[:2], good[:2])
    c.kv_lens.copy_(keep_lens)
    c.kv_lens[2] = -4  # no keys
    o, l = _call(c, q, [1, 1, 1], torch.float32)
    assert bool((o[2] == 0).all()) and bool((l[2] == -math.inf).all())
    c.kv_lens.copy_(keep_lens)
    plan = B.PagedPlan(3, 3, 4, 2, 64, ragged=True, q8=True)
    k, v, scales = c.tensors()
    for cu in ([0, 2, 1, 3], [1, 1, 2, 3], [0, 1, 2, 4], [0, -1, 2, 3]):
        o = torch.zeros_like(q)
        plan.run(q, k, v, o, c.kv_lens, c.table,
                 cu_q=torch.tensor(cu, dtype=torch.int32, device="cuda"), **scales)
        assert bool(torch.isnan(o).all()), cu


@pytest.mark.parametrize("ql,hq,hkv", [(2, 4, 1), (4, 8, 1), (60, 4, 2)])
def test_a_bad_page_shows_in_the_rows_that_need_it(ql, hq, hkv):
    """Rows of one row tile on both sides of a page that is none: the earlier
    ones do not keep its keys."""
    n, page = 64 + ql // 2, 16
    c = Cache8([n, 40], hkv, 64, page, seed=19)
    q = _q(2 * ql, hq, 64, 19)
    ref = c.reference(q, [ql, ql], 0.125)
    c.table[0, 64 // page] = -1
    o, l = _call(c, q, [ql, ql], torch.float32, ragged=True)
    first = ql - ql // 2  # the row at position 64
    assert bool(torch.isnan(o[first:ql]).all()) and bool(torch.isnan(l[first:ql]).all())
    rest = torch.cat([torch.arange(first), torch.arange(ql, 2 * ql)]).cuda()
    check(o[rest], l[rest], tuple(x[rest] for x in ref), torch.float32, f"bad page {ql}")


def test_bad_prefix_page_shows():
    c = Cache8([20, 30], 1, 64, 16, prefix=50, seed=4)
    q = _q(2, 4, 64, 10)
    c.prefix_pages[2] = c.k.shape[0]
    o, l = _call(c, q, [1, 1])
    assert bool(torch.isnan(o).all()) and bool(torch.isnan(l).all())


@pytest.mark.parametrize("ql", [1, 40])
def test_slopes_of_either_sign(ql):
    """Scores that grow with the distance, fall with it, or do not change."""
    sl = torch.tensor([-0.1, 0.0, 0.05, -0.01, 0.5, -0.03, 1.0, 0.2], device="cuda")
    c = Cache8([700, 90], 2, 64, 16, prefix=130, seed=17)
    q = _q(2 * ql, 8, 64, 18)
    o, l = _call(c, q, [ql, ql], torch.float32, None, sl, ragged=ql > 1)
    check(o, l, c.reference(q, [ql, ql], 0.125, None, sl), torch.float32, f"signs {ql}")


def test_same_bits_again_and_on_other_streams():
    """The same call again, on another stream, and two plans at once."""
    c = Cache8([5000, 40, 2000], 2, 128, 16, prefix=500, seed=16)
    k, v, scales = c.tensors()
    args = dict(prefix_pages=c.prefix_pages, prefix_len=500, **scales)
    side, calls = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i in range(2):
        q = _q(3, 8, 128, 30 + i)
        plan = B.PagedPlan(3, 3, 8, 2, 128, prefix=True, q8=True)
        want = torch.empty_like(q)
        plan.run(q, k, v, want, c.kv_lens, c.table, **args)
        again, _ = _call(c, q, [1] * 3)
        assert torch.equal(want, again)
        calls.append((q, plan, want, [torch.zeros_like(q) for _ in range(8)]))
    torch.cuda.synchronize()
    for j in range(8):
        for (q, plan, _, outs), stream in zip(calls, side):
            plan.run(q, k, v, outs[j], c.kv_lens, c.table, stream=stream, **args)
    torch.cuda.synchronize()
    for _, _, want, outs in calls:
        assert all(torch.equal(o, want) for o in outs)


def test_captured_calls_follow_lengths_and_share_a_plan():
    """Two captured calls of one plan in turn, lengths changed between."""
    lens = [700, 33, 64]
    c = Cache8(lens, 2, 64, 16, prefix=40, seed=13)
    k, v, scales = c.tensors()
    plan = B.PagedPlan(3, 3, 8, 2, 64, prefix=True, q8=True)
    args = dict(prefix_pages=c.prefix_pages, prefix_len=40, **scales)
    calls = []
    for i in range(2):
        q = _q(3, 8, 64, 13 + i)
        o = torch.zeros_like(q)
        plan.run(q, k, v, o, c.kv_lens, c.table, **args)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.run(q, k, v, o, c.kv_lens, c.table, **args)
        calls.append((q, o, graph))
    for now in ([700, 33, 64], [1, 33, 50], [650, 0, 17], [0, 0, 0], [699, 32, 64]):
        c.kv_lens.copy_(torch.tensor(now, dtype=torch.int32))
        c.lens = now
        for q, o, graph in calls:
            o.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            got = o.clone()
            fresh = torch.empty_like(o)
            B.PagedPlan(3, 3, 8, 2, 64, prefix=True, q8=True).run(q, k, v, fresh, c.kv_lens,
                                                                  c.table, **args)
            check(got, None, c.reference(q, [1] * 3, 0.125), torch.bfloat16, f"replay {now}")
            assert torch.equal(got, fresh)


def test_offsets_past_32_bits():
    """Pages whose byte offset in the cache passes 2^32, and scales past 2^25."""
    page, hkv, d = 256, 8, 128
    pages = 17000  # 17000 * 8 * 256 * 128 bytes = 4.5e9
    c = Cache8([600, 300], hkv, d, page, seed=15, spare=0)
    q = _q(2, 16, d, 15)
    want, wl = _call(c, q, [1, 1])
    ids = torch.tensor([16999, 8097, 16500, 2, 16998], device="cuda")
    for name in ("k8", "ks", "v8", "vs"):
        x = getattr(c, name)
        big = torch.zeros(pages, *x.shape[1:], dtype=torch.uint8, device="cuda")
        big[ids] = x
        setattr(c, name, big)
    c.table = torch.where(c.table >= 0, ids[c.table.clamp(min=0).long()].to(torch.int32), -1)
    got, gl = _call(c, q, [1, 1])
    assert torch.equal(got, want) and torch.equal(gl, wl)
    # a piece too
    q = _q(500, 16, d, 16)
    got, gl = _call(c, q, [300, 200], torch.float32)
    c.k, c.v = torch.zeros(0), torch.zeros(0)
    del big
    small = Cache8([600, 300], hkv, d, page, seed=15, spare=0)
    want, wl = _call(small, q, [300, 200], torch.float32)
    assert torch.equal(got, want) and torch.equal(gl, wl)


@pytest.mark.parametrize("form,d,ql,n,prefix", [
    ("two waves", 128, [1], 70001, 0), ("four waves", 64, [100], 33001, 0),
    ("two waves, 32 rows", 64, [20], 140001, 0), ("eight waves", 128, [200], 33001, 0),
    ("prefix, two waves", 128, [1] * 20, 40, 70001),
    ("prefix, four waves", 64, [1] * 40, 40, 33001)])
@pytest.mark.parametrize("score", ["plain", "slopes"])
@pytest.mark.parametrize("odd", [False, True])
def test_every_form_past_the_held_ids(form, d, ql, n, prefix, score, odd):
    """Shares of more pages than a workgroup holds ids for at a time, from the
    first key on and (with slopes) from the last one on; with `odd` also the
    pass that looks at masked values key by key.  Few pages under many ids."""
    heads, batch = 128, len(ql)
    c = Cache8([16 * 90], heads, d, 16, seed=25, spare=0)
    g = torch.Generator().manual_seed(26)
    far = max(n, prefix)
    ids = torch.randint(0, 88, (-(-far // 16),), generator=g).to(torch.int32)
    ids[-1] = 88  # the last page is its own: keys up to far, then NaN
    for name in ("k", "v"):
        getattr(c, name + "8")[88, :, far % 16:] = 255
        getattr(c, name + "s")[88, :, far % 16:] = 255
        getattr(c, name)[88, :, far % 16:] = math.nan
    own = torch.randint(0, 88, (batch, -(-n // 16)), generator=g).to(torch.int32)
    if prefix:
        c.prefix, c.prefix_pages = prefix, ids.cuda()
    else:
        own = ids[None].repeat(batch, 1)
    c.table, c.lens = own.cuda(), [n] * batch
    c.kv_lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    if odd and far % 16 > 1:
        c.v8[88, :, (far - 2) % 16, 5] = 127
        c.v[88, :, (far - 2) % 16, 5] = math.nan
    elif odd:  # the page before the last, which is then its own too
        ids[-2] = 89
        if prefix:
            c.prefix_pages = ids.cuda()
        else:
            c.table = ids[None].repeat(batch, 1).cuda()
        c.v8[89, :, 15, 5] = 127
        c.v[89, :, 15, 5] = math.nan
    sl = None
    if score == "slopes":  # flat, so that every segment weighs
        sl = torch.linspace(-2e-4, 2e-4, heads, device="cuda")
    q = _q(sum(ql), heads, d, 27)
    o, l = _call(c, q, ql, torch.float32, None, sl, ragged=max(ql) > 1)
    some = [0, 77, 127]
    c.k, c.v = c.k[:, some], c.v[:, some]
    check(o[:, some], l[:, some], c.reference(q[:, some], ql, d ** -0.5, None,
                                              sl[some] if sl is not None else None),
          torch.float32, f"{form} {score} {odd}")


@pytest.mark.parametrize("seed", range(10))
def test_shares_that_end_anywhere(seed):
    """Random lengths: shares end within row tiles, between them, and within
    what a row tile is charged beside its steps."""
    rng = random.Random(seed)
    d, hkv = rng.choice([64, 128]), rng.choice([1, 2, 8, 32])
    hq, page = hkv * rng.choice([1, 2, 4, 7]), rng.choice([16, 32, 256])
    batch = rng.choice([1, 3, 17, 70])
    lens = [rng.choice([0, 1, 64, 127, 128, 129, 300, rng.randrange(1, 4000)])
            for _ in range(batch)]
    prefix = rng.choice([0, 0, 200])
    c = Cache8(lens, hkv, d, page, prefix, seed=seed)
    ql = [1] * batch
    if seed % 3 == 2:
        ql = [rng.randrange(0, 5) for _ in range(batch)]
    q = _q(sum(ql), hq, d, seed)
    o, l = _call(c, q, ql, torch.float32, None, None, ragged=seed % 3 > 0)
    check(o, l, c.reference(q, ql, d ** -0.5), torch.float32, f"seed {seed}")
