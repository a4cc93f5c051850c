"""GPU tests of attention over the paged cache, against 64 bits."""
import math

import pytest
import torch

from paper_2507_21526_amd import binding as B
from tests.serving_ref import Cache, check, geometric_slopes

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
    plan = plan or B.PagedPlan(len(q_lens), total, hq, c.k.shape[1], d, prefix=c.prefix > 0,
                               ragged=ragged)
    plan.workspace.fill_(0xff)  # NaN bit patterns
    o = torch.full(q.shape, 7.0, dtype=dtype, device=q.device)
    l = torch.full((hq, total), 7.0, device=q.device) if lse else None
    plan.run(q, c.k, c.v, o, c.kv_lens, c.table, cu_q=cu,
             prefix_pages=c.prefix_pages if c.prefix else None, prefix_len=c.prefix, lse=l,
             softcap=softcap, slopes=slopes)
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
]


@pytest.mark.parametrize("case", SINGLE, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}-{c[2]}-"
                         f"{c[3]}-{c[4]}-{c[5]}")
@pytest.mark.parametrize("score", ["plain", "cap", "slopes", "both"])
def test_single_tokens(case, score):
    lens, hq, hkv, d, page, prefix = case
    c = Cache(lens, hkv, d, page, prefix, seed=len(lens) + hq)
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
]


@pytest.mark.parametrize("case", RAGGED, ids=lambda c: f"{max(c[0])}-{max(c[1])}-{c[2]}-{c[3]}-"
                         f"{c[4]}-{c[5]}-{c[6]}")
@pytest.mark.parametrize("score", ["plain", "both"])
def test_several_tokens(case, score):
    lens, ql, hq, hkv, d, page, prefix, behind = case
    c = Cache(lens, hkv, d, page, prefix, seed=hq)
    q = _q(sum(ql) + behind, hq, d, 6)
    cap, sl = (20.0, geometric_slopes(hq)) if score == "both" else (None, None)
    dtype = torch.bfloat16 if score == "both" else torch.float32
    o, l = _call(c, q, ql, dtype, cap, sl, ragged=True, behind=behind)
    ref = c.reference(q, ql, d ** -0.5, cap, sl)
    check(o, l, ref, dtype, f"{case} {score}")


def test_pages_past_the_held_ids():
    """A share of more pages than a workgroup holds ids for at a time: 128 kv
    heads leave two shares to a head."""
    c = Cache([20003], 128, 64, 16, seed=3)
    q = _q(1, 128, 64, 7)
    o, l = _call(c, q, [1], torch.float32)
    heads = [0, 77, 127]
    c.k, c.v = c.k[:, heads], c.v[:, heads]
    check(o[:, heads], l[:, heads], c.reference(q[:, heads], [1], 0.125), torch.float32,
          "segments")


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_batch(d, ragged):
    lens = [(7 * i) % 90 for i in range(1024)]
    ql = [(i % 3) for i in range(1024)] if ragged else [1] * 1024
    c = Cache(lens, 1, d, 16, prefix=20, seed=8)
    q = _q(sum(ql), 2, d, 9)
    o, l = _call(c, q, ql, torch.float32)
    pick = list(range(0, 1024, 37)) + [1023]
    starts = [0]
    for n in ql:
        starts.append(starts[-1] + n)
    some = [i for i in pick if ql[i]]
    at = torch.cat([torch.arange(starts[i], starts[i + 1]) for i in some]).cuda()
    sub = Cache([1], 1, d, 16)
    sub.k, sub.v, sub.prefix, sub.prefix_pages = c.k, c.v, c.prefix, c.prefix_pages
    sub.lens, sub.table = [lens[i] for i in some], c.table[some]
    check(o[at], l[at], sub.reference(q[at], [ql[i] for i in some], d ** -0.5), torch.float32,
          "1024 requests")


def test_many_row_tiles():
    """Near the limit of row tiles: a long piece of a prompt, many heads."""
    c = Cache([30000, 40], 1, 64, 256, seed=9)
    q = _q(30000 + 2, 8, 64, 10)
    o, l = _call(c, q, [30000, 2], ragged=True)
    rows = torch.cat([torch.arange(0, 30000, 1777), torch.tensor([29999])]).cuda()
    k, v = c.keys(0)
    dist = rows[:, None] - torch.arange(30000, device="cuda")
    from tests.serving_ref import attend
    check(o[rows], l[rows], attend(q[rows], k, v, dist >= 0, dist, 0.125), torch.bfloat16, "piece")
    c.lens, c.table = [40], c.table[1:]
    check(o[30000:], l[30000:], c.reference(q[30000:], [2], 0.125), torch.bfloat16, "two rows")


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d,ql", [(64, 4), (128, 4), (128, 50)])
def test_values_behind_a_row(bad, d, ql):
    """An infinite or NaN value reaches the rows that keep its key, and no
    other: neither earlier rows of the same call nor later requests."""
    lens = [150, 60]
    c = Cache(lens, 1, d, 16, seed=1)
    q = _q(2 * ql, 4, d, 8)
    for b, back in ((0, 2), (1, 1)):  # the last but one key, the last key
        p = lens[b] - back
        page = int(c.table[b, p // 16])
        c.v[page, 0, p % 16, 3] = bad
        c.v[page, 0, p % 16, d - 1] = bad
    o, l = _call(c, q, [ql, ql], torch.float32, ragged=True)
    ref = c.reference(q, [ql, ql], d ** -0.5)
    keeps = ~torch.isfinite(ref[0]).all(-1).all(-1)
    assert int(keeps.sum()) == 3  # two rows of the first request, one of the second
    check(o, l, ref, torch.float32, f"{bad} d {d} rows {ql}")


@pytest.mark.parametrize("hq,d", [(1, 128), (1, 64), (3, 128), (8, 64)])
def test_values_in_every_part_of_a_step(hq, d):
    """Rows of one head or few: at one step some waves of a row tile drop keys
    and others keep all of them.  A value of each key in turn is infinite; no
    row before the key sees it."""
    n = 128
    c = Cache([n], 1, d, 16, seed=5)
    q = _q(n, hq, d, 12)
    clean, _ = _call(c, q, [n], torch.float32, ragged=True)
    keep = c.v.clone()
    for j in range(0, n, 3):
        c.v.copy_(keep)
        c.v[int(c.table[0, j // 16]), 0, j % 16, j % d] = math.inf
        o, _ = _call(c, q, [n], torch.float32, ragged=True)
        assert bool(torch.isfinite(o[:j]).all()), j
        # the same sums, key by key: bits may differ by their order
        assert float((o[:j] - clean[:j]).abs().max() if j else 0.0) < 1e-5, j
        assert not bool(torch.isfinite(o[j:, :, j % d]).any()), j


def test_bad_pages_and_lengths_show():
    """A page id outside the cache, and a length past the table, give NaN in
    the rows of that request and nowhere else; bad query offsets in all."""
    lens = [100, 90, 80]
    c = Cache(lens, 2, 64, 16, seed=2)
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
    plan = B.PagedPlan(3, 3, 4, 2, 64, ragged=True)
    for cu in ([0, 2, 1, 3], [1, 1, 2, 3], [0, 1, 2, 4], [0, -1, 2, 3]):
        o = torch.zeros_like(q)
        plan.run(q, c.k, c.v, o, c.kv_lens, c.table,
                 cu_q=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        assert bool(torch.isnan(o).all()), cu


def test_bad_prefix_page_shows():
    c = Cache([20, 30], 1, 64, 16, prefix=50, seed=4)
    q = _q(2, 4, 64, 10)
    c.prefix_pages[2] = c.k.shape[0]
    o, l = _call(c, q, [1, 1])
    assert bool(torch.isnan(o).all()) and bool(torch.isnan(l).all())


def test_prefix_equals_the_same_keys_in_own_pages():
    """A shared prefix gives what the same keys at the front of every
    request's own pages give, up to rounding."""
    page, pre, lens = 16, 96, [33, 1, 200]
    c = Cache(lens, 2, 128, page, pre, seed=11)
    q = _q(3, 8, 128, 11)
    sl = geometric_slopes(8)
    o, l = _call(c, q, [1] * 3, torch.float32, 9.0, sl)
    n = pre // page
    flat = Cache([1], 2, 128, page, seed=0)
    flat.k, flat.v, flat.prefix, flat.page = c.k, c.v, 0, page
    flat.table = torch.cat([c.prefix_pages[None].expand(3, n), c.table], 1).contiguous()
    flat.lens = [pre + x for x in lens]
    flat.kv_lens = c.kv_lens + pre
    o2, l2 = _call(flat, q, [1] * 3, torch.float32, 9.0, sl)
    ref = c.reference(q, [1] * 3, 128 ** -0.5, 9.0, sl)
    check(o, l, ref, torch.float32, "prefix")
    check(o2, l2, ref, torch.float32, "own")


def test_same_bits_again_and_on_another_stream():
    c = Cache([3000, 17, 900], 2, 128, 16, prefix=333, seed=12)
    q = _q(3, 8, 128, 12)
    o, l = _call(c, q, [1] * 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, l2 = _call(c, q, [1] * 3)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(l, l2)
    plan = B.PagedPlan(3, 3, 8, 2, 128, prefix=True)
    o3 = torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    plan.run(q, c.k, c.v, o3, c.kv_lens, c.table, prefix_pages=c.prefix_pages,
             prefix_len=c.prefix, stream=side)
    side.synchronize()
    assert torch.equal(o, o3)


def test_two_calls_at_once():
    """Two plans on two streams, several calls in flight."""
    c = Cache([5000, 40, 2000], 2, 128, 16, prefix=500, seed=16)
    side, calls = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i in range(2):
        q = _q(3, 8, 128, 30 + i)
        plan = B.PagedPlan(3, 3, 8, 2, 128, prefix=True)
        want = torch.empty_like(q)
        plan.run(q, c.k, c.v, want, c.kv_lens, c.table, prefix_pages=c.prefix_pages,
                 prefix_len=500)
        calls.append((q, plan, want, [torch.zeros_like(q) for _ in range(8)]))
    torch.cuda.synchronize()
    for j in range(8):
        for (q, plan, _, outs), stream in zip(calls, side):
            plan.run(q, c.k, c.v, outs[j], c.kv_lens, c.table, prefix_pages=c.prefix_pages,
                     prefix_len=500, stream=stream)
    torch.cuda.synchronize()
    for _, _, want, outs in calls:
        assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("ql", [1, 40])
def test_slopes_of_either_sign(ql):
    """Scores that grow with the distance, fall with it, or do not change."""
    sl = torch.tensor([-0.1, 0.0, 0.05, -0.01, 0.5, -0.03, 1.0, 0.2], device="cuda")
    c = Cache([700, 90], 2, 64, 16, prefix=130, seed=17)
    q = _q(2 * ql, 8, 64, 18)
    o, l = _call(c, q, [ql, ql], torch.float32, None, sl, ragged=ql > 1)
    check(o, l, c.reference(q, [ql, ql], 0.125, None, sl), torch.float32, f"signs {ql}")


def test_captured_call_follows_lengths_and_tables():
    lens = [700, 33, 64]
    c = Cache(lens, 2, 64, 16, seed=13)
    q = _q(3, 8, 64, 13)
    plan = B.PagedPlan(3, 3, 8, 2, 64)
    o = torch.zeros_like(q)
    plan.run(q, c.k, c.v, o, c.kv_lens, c.table)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run(q, c.k, c.v, o, c.kv_lens, c.table)
    for now in ([700, 33, 64], [1, 33, 50], [650, 0, 17], [0, 0, 0], [699, 32, 64]):
        c.kv_lens.copy_(torch.tensor(now, dtype=torch.int32))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        fresh = torch.empty_like(o)
        B.PagedPlan(3, 3, 8, 2, 64).run(q, c.k, c.v, fresh, c.kv_lens, c.table)
        c.lens = now
        ref = c.reference(q, [1] * 3, 0.125)
        check(got, None, ref, torch.bfloat16, f"replay {now}")
        assert torch.equal(got, fresh)


def test_two_graphs_of_one_plan_in_turn():
    """Two captured calls of one plan share its workspace: in turn on one
    stream each gives its own result."""
    c = Cache([2000, 90], 1, 128, 16, prefix=200, seed=14)
    plan = B.PagedPlan(2, 2, 4, 1, 128, prefix=True)
    calls = []
    for i in range(2):
        q, o = _q(2, 4, 128, 20 + i), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda")
        args = dict(prefix_pages=c.prefix_pages, prefix_len=200)
        plan.run(q, c.k, c.v, o, c.kv_lens, c.table, **args)
        torch.cuda.synchronize()
        want, graph = o.clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.run(q, c.k, c.v, o, c.kv_lens, c.table, **args)
        calls.append((graph, o, want, q))  # q is read by every replay
    for _ in range(3):
        for graph, o, want, _q_kept in calls:
            o.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want)
        torch.zeros(1000, device="cuda").add_(1)


def test_offsets_past_32_bits():
    """Pages whose byte offset in the cache passes 2^32 (and element offset
    2^31)."""
    page, hkv, d = 256, 8, 128
    pages = 9000  # 9000 * 8 * 256 * 128 * 2 bytes = 4.7e9
    k = torch.zeros(pages, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    c = Cache([600, 300], hkv, d, page, seed=15, spare=0)
    ids = torch.tensor([8999, 4097, 8500, 2, 8998], device="cuda")
    k[ids], v[ids] = c.k, c.v
    small = c.k, c.v, c.table.clone()
    q = _q(2, 16, d, 15)
    want, wl = _call(c, q, [1, 1])
    c.k, c.v = k, v
    c.table = torch.where(c.table >= 0, ids[c.table.clamp(min=0).long()].to(torch.int32), -1)
    got, gl = _call(c, q, [1, 1])
    assert torch.equal(got, want) and torch.equal(gl, wl)
    # and the write that fills such pages
    rows = torch.randn(5, hkv, d, device="cuda").bfloat16()
    slots = torch.tensor([8999 * 256 + 255, 4097 * 256, -1, 8500 * 256 + 17, pages * 256],
                         dtype=torch.int32, device="cuda")
    B.kv_cache_write(rows, -rows, slots, k, v)
    for i, s in ((0, 8999 * 256 + 255), (1, 4097 * 256), (3, 8500 * 256 + 17)):
        assert torch.equal(k[s // 256, :, s % 256], rows[i])
        assert torch.equal(v[s // 256, :, s % 256], -rows[i])
    del small


@pytest.mark.parametrize("ql,hq,hkv", [(2, 4, 1), (4, 8, 1), (60, 4, 2)])
def test_a_bad_page_shows_in_the_rows_that_need_it(ql, hq, hkv):
    """Rows of one row tile on both sides of a page that is none: the earlier
    ones do not keep its keys."""
    n, page = 64 + ql // 2, 16
    c = Cache([n, 40], hkv, 64, page, seed=19)
    q = _q(2 * ql, hq, 64, 19)
    ref = c.reference(q, [ql, ql], 0.125)
    c.table[0, 64 // page] = -1
    o, l = _call(c, q, [ql, ql], torch.float32, ragged=True)
    first = ql - ql // 2  # the row at position 64
    assert bool(torch.isnan(o[first:ql]).all()) and bool(torch.isnan(l[first:ql]).all())
    rest = torch.cat([torch.arange(first), torch.arange(ql, 2 * ql)]).cuda()
    check(o[rest], l[rest], tuple(x[rest] for x in ref), torch.float32, f"bad page {ql}")


def _equal_far_keys(c, hq, places):
    """Queries of one direction, and keys whose products make up for the bias
    of slope -4 at these places from the first key (of the prefix): their
    scores are equal, all others far below.  bf16 holds 2 x these places."""
    c.k.zero_()
    for j in places:
        if j < c.prefix:
            page, at = int(c.prefix_pages[j // c.page]), j % c.page
        else:
            page, at = int(c.table[0, (j - c.prefix) // c.page]), (j - c.prefix) % c.page
        c.k[page, :, at, 0] = 2.0 * j  # 0.125 * 16 * 2 j = 4 j
    return torch.full((hq,), -4.0, device="cuda")


@pytest.mark.parametrize("d,ql,prefix", [(64, 1, 0), (64, 5, 0), (128, 40, 0), (64, 1, 300),
                                         (128, 7, 300)])
def test_scores_that_grow_over_far_distances(d, ql, prefix):
    """Biases of 280000 between a row and the keys that it attends to, some
    tiles apart, in the prefix and behind it: equal scores stay equal."""
    c = Cache([70001], 1, d, 256, prefix=prefix, seed=20)
    c.v.nan_to_num_()
    sl = _equal_far_keys(c, 2, [0, 70, 140, 210, 350])
    q = torch.zeros(ql, 2, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 16.0
    plan = B.PagedPlan(1, ql, 2, 1, d, prefix=prefix > 0, ragged=True)
    cu = torch.tensor([0, ql], dtype=torch.int32, device="cuda")
    o, l = torch.empty(ql, 2, d, device="cuda"), torch.empty(2, ql, device="cuda")
    plan.run(q, c.k, c.v, o, c.kv_lens, c.table, cu_q=cu,
             prefix_pages=c.prefix_pages if prefix else None, prefix_len=prefix, lse=l,
             softmax_scale=0.125, slopes=sl)
    check(o, l.t(), c.reference(q, [ql], 0.125, None, sl), torch.float32, f"far {d} {ql} {prefix}")


@pytest.mark.parametrize("form,d,ql,n,prefix", [
    ("two waves", 128, [1], 33001, 0), ("four waves", 64, [100], 33001, 0),
    ("prefix, two waves", 128, [1] * 20, 40, 33001),
    ("prefix, four waves", 64, [1] * 40, 40, 33001)])
@pytest.mark.parametrize("score", ["plain", "slopes"])
@pytest.mark.parametrize("odd", [False, True])
def test_every_form_past_the_held_ids(form, d, ql, n, prefix, score, odd):
    """Shares of more pages than a workgroup holds ids for at a time, from the
    first key on and (with slopes) from the last one on; with `odd` also the
    pass that looks at masked values key by key.  Few pages under many ids."""
    heads, batch = 128, len(ql)
    c = Cache([16 * 90], heads, d, 16, seed=25, spare=0)
    g = torch.Generator().manual_seed(26)
    far = max(n, prefix)
    ids = torch.randint(0, 88, (-(-far // 16),), generator=g).to(torch.int32)
    ids[-1] = 88  # the last page is its own: 9 keys, then NaN
    c.k[88, :, far % 16:] = math.nan
    c.v[88, :, far % 16:] = math.nan
    own = torch.randint(0, 88, (batch, -(-n // 16)), generator=g).to(torch.int32)
    if prefix:
        c.prefix, c.prefix_pages = prefix, ids.cuda()
    else:
        own = ids[None].repeat(batch, 1)
    c.table, c.lens = own.cuda(), [n] * batch
    c.kv_lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    if odd:
        c.v[88, :, (far - 2) % 16, 5] = math.inf
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
