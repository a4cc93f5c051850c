"""GPU tests of prefill attention with modified scores, against 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2507_21526_amd import binding as B
from paper_2507_21526_amd.inputs import draw_qkv
from tests.serving_ref import attend, check, geometric_slopes, scored_keep

pytestmark = pytest.mark.gpu


def _lists(cu, tile, seed):
    """Per-q-tile lists of every sequence, some of them empty."""
    rng = np.random.default_rng(seed)
    ptr, idx, per = [0], [], []
    for a, b in zip(cu, cu[1:]):
        mine = []
        for t in range(-(-(b - a) // tile)):
            tiles = [] if t % 5 == 3 else sorted(
                set(np.flatnonzero(rng.random(t + 1) < 0.5).tolist()) | ({t} if t % 2 else set()))
            mine.append(tiles)
            idx.extend(tiles)
            ptr.append(len(idx))
        per.append(mine)
    return (ptr, idx), per


def _run(kind, cu, hq, hkv, d, tile, S, W, L, cap, slopes, dtype, splits=0, seed=1, blocks=None,
         qkv=None):
    q, k, v = qkv or (t.cuda() for t in draw_qkv(cu, hq, hkv, d, seed, key0_boost=8.0))
    plan = B.Plan(kind, cu, S, W, L, tile, hq, d, splits, blocks=blocks)
    if plan.workspace is not None:
        plan.workspace.fill_(0xff)
    o = torch.full(q.shape, math.nan, dtype=dtype, device="cuda")
    lse = torch.full((hq, cu[-1]), math.nan, device="cuda")
    plan.run(q, k, v, o, lse, softcap=cap, slopes=slopes)
    torch.cuda.synchronize()
    return q, k, v, o, lse, plan


def _verify(kind, cu, q, k, v, o, lse, tile, S, W, L, cap, slopes, label, lists=None, rows=None,
            underflow=False):
    for i, (a, b) in enumerate(zip(cu, cu[1:])):
        n = b - a
        if n == 0:
            continue
        keep = torch.from_numpy(scored_keep(kind, n, S, W, L, tile,
                                            lists[i] if lists else None)).cuda()
        pick = torch.arange(n, device="cuda") if rows is None else rows(n)
        dist = pick[:, None] - torch.arange(n, device="cuda")
        ref = attend(q[a:b][pick], k[a:b], v[a:b], keep[pick], dist, q.shape[2] ** -0.5, cap,
                     slopes)
        check(o[a:b][pick], lse[:, a:b].t()[pick], ref, o.dtype, f"{label} sequence {i}",
              underflow)


CASES = [
    # kind, cu, hq, hkv, d, tile, S, W, L, splits
    ("causal", [0, 1], 1, 1, 64, 64, 0, 1, 0, 0),
    ("causal", [0, 63, 64, 64, 193, 450], 4, 1, 128, 128, 0, 1, 0, 0),
    ("causal", [0, 333], 7, 1, 64, 64, 0, 1, 0, 0),
    ("causal", [0, 700], 10, 2, 128, 64, 0, 1, 0, 0),
    ("triangle", [0, 300], 4, 1, 64, 64, 8, 64, 20, 0),
    ("triangle", [0, 900, 901, 1000], 8, 1, 128, 128, 8, 200, 40, 0),
    ("triangle", [0, 1300], 6, 2, 128, 128, 128, 256, 128, 7),
    ("triangle", [0, 800], 3, 1, 64, 128, 0, 130, 0, 0),       # no sink, no Last rows
    ("triangle", [0, 777], 5, 1, 128, 64, 70, 1, 3, 0),        # a window of one key
    ("triangle", [0, 640], 16, 2, 64, 64, 100, 90, 640, 5),    # every row is a Last row
    ("blocksparse", [0, 700, 1100], 4, 2, 128, 64, 0, 1, 0, 2),
    ("blocksparse", [0, 900], 8, 1, 64, 128, 0, 1, 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1][-1]}-{c[2]}-{c[3]}-{c[4]}-"
                         f"{c[5]}-{c[6]}-{c[7]}-{c[8]}")
@pytest.mark.parametrize("score", ["cap", "slopes", "both"])
def test_parity(case, score):
    kind, cu, hq, hkv, d, tile, S, W, L, splits = case
    cap = 11.0 if score != "slopes" else None
    sl = geometric_slopes(hq) if score != "cap" else None
    dtype = torch.float32 if score == "slopes" else torch.bfloat16
    blocks, per = _lists(cu, tile, 3) if kind == "blocksparse" else (None, None)
    q, k, v, o, lse, plan = _run(kind, cu, hq, hkv, d, tile, S, W, L, cap, sl, dtype, splits,
                                 blocks=blocks)
    _verify(kind, cu, q, k, v, o, lse, tile, S, W, L, cap, sl, f"{case} {score}", per)


def test_long_triangle_and_causal_rows():
    """Sampled rows of long sequences: split Last rows, far distances."""
    def rows(n):
        g = torch.Generator().manual_seed(n)
        r = torch.cat([torch.randint(0, n, (40,), generator=g), torch.tensor(
            [0, 127, 128, n - 129, n - 128, n - 1])])
        return r.unique().cuda()

    for kind, n, cap, slopes in (("triangle", 9000, None, geometric_slopes(8) / 16),
                                 ("causal", 5000, 30.0, None)):
        cu = [0, n]
        out = _run(kind, cu, 8, 2, 128, 128, 128, 1024, 128, cap, slopes, torch.float32)
        _verify(kind, cu, *out[:5], 128, 128, 1024, 128, cap, slopes, f"long {kind}", rows=rows)


@pytest.mark.parametrize("kind", ["causal", "triangle"])
def test_slopes_of_either_sign(kind):
    """Scores that grow with the distance, fall with it, or do not change."""
    sl = torch.tensor([-0.1, 0.0, 0.05, -0.01, 0.5, -0.03, 1.0, 0.2], device="cuda")
    cu = [0, 600, 777]
    out = _run(kind, cu, 8, 2, 128, 128, 8, 100, 30, None, sl, torch.float32)
    _verify(kind, cu, *out[:5], 128, 8, 100, 30, None, sl, f"signs {kind}")


def test_a_cap_of_zero_is_none():
    cu = [0, 300]
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, 64, 3))
    plan = B.Plan("causal", cu, 0, 1, 0, 64, 4, 64)
    a, b = torch.empty_like(q), torch.empty_like(q)
    plan.run(q, k, v, a)
    plan.run(q, k, v, b, softcap=0.0)
    assert torch.equal(a, b)


def test_a_wide_cap_and_no_slope_are_the_plain_pass():
    """Slopes of zero change nothing but the order of roundings."""
    cu = [0, 500, 800]
    q, k, v, o, lse, plan = _run("triangle", cu, 8, 2, 128, 128, 8, 100, 30, None,
                                 torch.zeros(8, device="cuda"), torch.float32)
    po, pl = torch.empty_like(o), torch.empty_like(lse)
    plan.run(q, k, v, po, pl)
    torch.cuda.synchronize()
    assert float((o - po).norm() / po.norm()) < 2 * 2.0 ** -8  # each rounds P to bf16
    assert float((lse - pl).abs().max()) < 2 * 2.0 ** -13


@pytest.mark.parametrize("cap", [0.5, 50.0, 1000.0])
def test_cap_holds_far_scores(cap):
    """Scores far past the cap, both signs: keys of 100 times the norm."""
    cu = [0, 200]
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, 64, 9))
    k[::3] *= 100
    q, k, v, o, lse, _ = _run("causal", cu, 4, 1, 64, 64, 0, 1, 0, cap, None, torch.float32,
                              qkv=(q, k, v))
    dist = torch.arange(200, device="cuda")[:, None] - torch.arange(200, device="cuda")
    ro, rl, absw = attend(q, k, v, dist >= 0, dist, 0.125, cap)
    # products of up to 100 * 30: an error e of a product is damped by the
    # tanh's slope, at most e; 3000 * 2^-24 * 16 = 2.9e-3, and 2^-22 cap
    e = 2.9e-3 + 2.0 ** -22 * cap
    assert bool(((o.double() - ro).abs() <= (2.0 ** -8 + 2 * e) * absw + 1e-5).all())
    assert bool(((lse.t().double() - rl).abs() <= e + 2.0 ** -22 * rl.abs()).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("kind,d,W", [("causal", 128, 1), ("triangle", 64, 70)])
def test_values_of_masked_keys(bad, kind, d, W):
    """An infinite or NaN value reaches the rows that keep its key only, also
    within a step of keys."""
    cu = [0, 300]
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, d, 10))
    for j in (100, 150, 299):
        v[j, 0, 5] = bad
    out = _run(kind, cu, 4, 1, d, 64, 0, W, 0, 20.0, None, torch.float32, qkv=(q, k, v))
    _verify(kind, cu, *out[:5], 64, 0, W, 0, 20.0, None, f"{kind} {bad}")


@pytest.mark.parametrize("hq,d,tile", [(1, 128, 128), (1, 64, 128), (3, 128, 128), (2, 64, 64)])
def test_values_in_every_part_of_a_step(hq, d, tile):
    """Waves of one workgroup with other rows: at one step some drop keys and
    others keep all of them."""
    n = 128
    q, k, v = (t.cuda() for t in draw_qkv([0, n], hq, 1, d, 13))
    args = ("causal", [0, n], hq, 1, d, tile, 0, 1, 0, 20.0, None, torch.float32)
    clean = _run(*args, qkv=(q, k, v))[3]
    for j in range(0, n, 3):
        w = v.clone()
        w[j, 0, j % d] = math.inf
        o = _run(*args, qkv=(q, k, w))[3]
        assert bool(torch.isfinite(o[:j]).all()), j
        assert float((o[:j] - clean[:j]).abs().max() if j else 0.0) < 1e-5, j
        assert not bool(torch.isfinite(o[j:, :, j % d]).any()), j


def test_infinite_keys_at_masked_places():
    """A NaN key that a row does not keep changes nothing for it."""
    cu = [0, 200]
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, 128, 12))
    sl = geometric_slopes(4)
    want = _run("causal", cu, 4, 1, 128, 64, 0, 1, 0, 15.0, sl, torch.float32, qkv=(q, k, v))[3]
    k2 = k.clone()
    k2[150:] = math.nan
    got = _run("causal", cu, 4, 1, 128, 64, 0, 1, 0, 15.0, sl, torch.float32, qkv=(q, k2, v))[3]
    assert torch.equal(got[:150], want[:150])
    assert bool(torch.isnan(got[150:]).all())


@pytest.mark.parametrize("kind", ["triangle", "causal", "blocksparse"])
def test_a_schedule_that_does_not_fit_shows(kind):
    cu = [0, 600]
    blocks, _ = _lists(cu, 64, 3)
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, 64, 2))
    plan = B.Plan(kind, cu, 8, 100, 64, 64, 4, 64, 2, blocks=blocks)
    o = torch.zeros(q.shape, device="cuda")
    lse = torch.zeros(4, 600, device="cuda")
    for word, value in ((0, 1), (2, 7), (3, 128), (11, 5)):  # magic, kind, tile, items
        keep = int(plan.sched[word])
        plan.sched[word] = value
        plan.run(q, k, v, o.zero_(), lse.zero_(), softcap=5.0)
        assert bool(torch.isnan(o).all()) and bool(torch.isnan(lse).all()), word
        plan.sched[word] = keep
    item = 16 + 12 * (plan.info.n_items - 1)  # the last item: its rows are its own
    r0, r1 = int(plan.sched[item + 2]), int(plan.sched[item + 3])
    part = int(plan.sched[item + 9])
    plan.sched[item + 8] = 9  # no such mode
    plan.run(q, k, v, o.zero_(), lse.zero_(), softcap=5.0)
    assert part >= 0 or bool(torch.isnan(o[r0:r1]).all())


def test_empty_batches_and_streams():
    for cu in ([0], [0, 0, 0]):
        q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
        k = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
        B.Plan("causal", cu, 0, 1, 0, 64, 4, 64).run(q, k, k.clone(), torch.empty_like(q),
                                                     softcap=5.0)
    cu = [0, 700]
    sl = geometric_slopes(4)
    q, k, v, o, lse, plan = _run("triangle", cu, 4, 1, 64, 64, 8, 100, 64, 9.0, sl,
                                 torch.bfloat16, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2 = torch.zeros_like(o)
    plan.run(q, k, v, o2, stream=side, softcap=9.0, slopes=sl)
    side.synchronize()
    assert torch.equal(o, o2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.run(q, k, v, o2, softcap=9.0, slopes=sl)
    for _ in range(3):
        o2.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o2)
        plan.run(q, k, v, torch.empty_like(o), softcap=9.0)


EIGHT = [
    # kind, cu, hq, hkv, tile, S, W, L: over 512 workgroups of eight waves
    ("causal", [0, 4500], 32, 8, 128, 0, 1, 0),
    ("causal", [0, 700, 701, 4500], 32, 4, 64, 0, 1, 0),  # (11 + 1 + 60) 2 4 = 576
    ("triangle", [0, 3001, 5200], 24, 8, 128, 70, 300, 100),  # a group of three: four waves
    ("triangle", [0, 3001, 5200], 32, 8, 128, 70, 300, 100),
    ("blocksparse", [0, 3000, 4700], 32, 8, 128, 0, 1, 0),
]


@pytest.mark.parametrize("case", EIGHT, ids=lambda c: f"{c[0]}-{c[1][-1]}-{c[2]}-{c[3]}-{c[4]}")
@pytest.mark.parametrize("score", ["cap", "slopes"])
@pytest.mark.parametrize("odd", [False, True])
def test_larger_launches(case, score, odd):
    """The eight-wave form (and, for a group that does not fill it, the
    four-wave one), also with infinite values in masked steps."""
    from tests.parity import kernels_of
    kind, cu, hq, hkv, tile, S, W, L = case
    cap, sl = (20.0, None) if score == "cap" else (None, geometric_slopes(hq))
    blocks, per = _lists(cu, tile, 4) if kind == "blocksparse" else (None, None)
    q, k, v = (t.cuda() for t in draw_qkv(cu, hq, hkv, 128, 21, key0_boost=8.0))
    if odd:
        for j in (cu[1] - 1, cu[-1] - 30, 100):
            v[j, 0, 7] = math.inf
    out = {}
    names = kernels_of(lambda: out.update(r=_run(
        kind, cu, hq, hkv, 128, tile, S, W, L, cap, sl, torch.bfloat16, blocks=blocks,
        qkv=(q, k, v))))
    waves = 8 if (hq // hkv * tile // 32) % 8 == 0 else 4
    assert any(f"{waves}>" in n for n in names if "scored_attn" in n), names
    q, k, v, o, lse, _ = out["r"]
    heads = [0, hq // hkv, hq - 1]

    def rows(n):
        g = torch.Generator().manual_seed(n)
        r = torch.cat([torch.randint(0, n, (50,), generator=g),
                       torch.tensor([0, n - 1, n // 2, max(0, n - 31)])])
        return r.unique().cuda()

    for h in heads:
        one = [h * hkv // hq]
        _verify(kind, cu, q[:, [h]], k[:, one], v[:, one], o[:, [h]], lse[[h]], tile, S, W, L, cap,
                sl[[h]] if sl is not None else None, f"{case} {score} {odd} head {h}", per, rows,
                underflow=odd and score == "slopes")


@pytest.mark.parametrize("sink", [2 ** 31 - 1, 2 ** 31 - 63, 2 ** 31 - 64])
@pytest.mark.parametrize("d,hq,last", [(128, 4, 0), (64, 3, 40)])
@pytest.mark.parametrize("score", ["cap", "slopes"])
def test_every_key_a_sink(sink, d, hq, last, score):
    """A sink longer than any sequence, up to the largest number: every row
    keeps all earlier keys."""
    cu = [0, 1000, 1013, 1300]
    cap, sl = (20.0, None) if score == "cap" else (None, geometric_slopes(hq))
    out = _run("triangle", cu, hq, 1, d, 64, sink, 64, last, cap, sl, torch.float32)
    _verify("triangle", cu, *out[:5], 64, sink, 64, last, cap, sl, f"sink {sink} {score}")


def test_every_key_a_sink_in_eight_waves():
    cu = [0, 4500]  # 36 items of 2 workgroups a kv head
    sl = geometric_slopes(32)
    qkv = tuple(t.cuda() for t in draw_qkv(cu, 32, 8, 128, 22))
    want = _run("triangle", cu, 32, 8, 128, 128, 4500, 128, 0, None, sl, torch.bfloat16, qkv=qkv)
    got = _run("triangle", cu, 32, 8, 128, 128, 2 ** 31 - 1, 128, 0, None, sl, torch.bfloat16,
               qkv=qkv)
    assert torch.equal(got[3], want[3]) and torch.equal(got[4], want[4])


@pytest.mark.parametrize("kind,d", [("causal", 64), ("causal", 128), ("triangle", 128),
                                    ("blocksparse", 64)])
def test_scores_that_grow_over_far_distances(kind, d):
    """Biases of 260000 between a row and the keys that it attends to, some
    steps apart: equal scores stay equal.  (0.125 * 16 * 2 j makes up for slope
    -4 at key j; bf16 holds these 2 j.)"""
    n, tile, sl = 66000, 128, torch.full((2,), -4.0, device="cuda")
    cu, blocks = [0, n], None
    if kind == "blocksparse":  # the first tiles, in some q-tiles cut in three
        lists = [list(range(min(t + 1, 3 if t % 2 else 40))) for t in range(-(-n // tile))]
        blocks = (np.cumsum([0] + [len(x) for x in lists]).tolist(), sum(lists, []))
    g = torch.Generator().manual_seed(23)
    q = torch.zeros(n, 2, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 16.0
    k = torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(n, 1, d, generator=g).bfloat16().cuda()
    places = torch.tensor([0, 70, 140, 210, 350], device="cuda")
    k[places, 0, 0] = 2.0 * places.to(torch.bfloat16)
    S, W, L = 360, 256, 200
    plan = B.Plan(kind, cu, S, W, L, tile, 2, d, 16 if kind == "blocksparse" else 0,
                  blocks=blocks)
    o, l = torch.empty(n, 2, d, device="cuda"), torch.empty(2, n, device="cuda")
    plan.run(q, k, v, o, l, softmax_scale=0.125, slopes=sl)
    rows = torch.cat([torch.arange(5000, n, 3001), torch.arange(n - 250, n, 7)]).cuda()
    key = torch.arange(n, device="cuda")
    keep = key <= rows[:, None]
    if kind == "triangle":
        keep &= (key < S) | (rows[:, None] - key < W) | (rows[:, None] >= n - L)
    if kind == "blocksparse":
        many = torch.where((rows // tile) % 2 == 1, 3, 40)
        keep &= key // tile < many[:, None]
    ref = attend(q[rows], k, v, keep, rows[:, None] - key, 0.125, None, sl)
    check(o[rows], l.t()[rows], ref, torch.float32, f"far {kind} {d}")


def test_scores_that_grow_within_a_window():
    """Without a sink a streaming row's first key is its window's."""
    n, W = 5000, 400
    q = torch.zeros(n, 2, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(n, 1, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(n, 1, 64, generator=torch.Generator().manual_seed(24)).bfloat16().cuda()
    q[..., 0] = 16.0
    row = 4700
    keys = row - W + 1 + torch.tensor([0, 50, 100, 150, 350], device="cuda")
    # 0.125 * 16 * k makes up for slope -512 from the window's start on
    k[keys, 0, 0] = 256.0 * (keys - keys[0]).to(torch.bfloat16)
    sl = torch.full((2,), -512.0, device="cuda")
    plan = B.Plan("triangle", [0, n], 0, W, 0, 64, 2, 64)
    o, l = torch.empty(n, 2, 64, device="cuda"), torch.empty(2, n, device="cuda")
    plan.run(q, k, v, o, l, softmax_scale=0.125, slopes=sl)
    at = torch.arange(n, device="cuda")
    rows = torch.cat([torch.arange(100), torch.arange(row - 2, row + 3)]).cuda()
    gap = rows[:, None] - at
    ref = attend(q[rows], k, v, (gap >= 0) & (gap < W), gap, 0.125, None, sl)
    # In the log2 domain products and biases are below 512 * 400 * 1.4427 < 2^19,
    # half a step of which is 2^-6: the tile's bias, its difference to the
    # reference and a key's own bias round by that each, the sum of product and
    # bias is small.  A probability is off by a factor of e^(+-e) at most, an
    # output by e^(2 e) - 1 beside the rounding of probabilities to bf16.
    e = 3 * 2.0 ** -6 * math.log(2.0)
    ro, rl, absw = ref
    assert bool(((o[rows].double() - ro).abs() <= (2.0 ** -8 + math.expm1(2 * e)) * absw
                 + 1e-5).all())
    assert bool(((l.t()[rows].double() - rl).abs() <= e + 2.0 ** -22 * rl.abs()).all())


@pytest.mark.parametrize("score", ["cap", "slopes"])
def test_lists_longer_than_a_workgroup_holds(score):
    """Items of more listed steps than a workgroup keeps in LDS."""
    n, tile = 64 * 2200 + 17, 64
    count = -(-n // tile)
    full = {count - 1, count - 3}  # two q-tiles list all earlier tiles
    lists = [list(range(t + 1)) if t in full else [t] for t in range(count)]
    blocks = (np.cumsum([0] + [len(x) for x in lists]).tolist(), sum(lists, []))
    cap = 20.0 if score == "cap" else None
    sl = torch.tensor([1e-5, -1e-5], device="cuda") if score == "slopes" else None
    cu = [0, n]
    q, k, v, o, lse, plan = _run("blocksparse", cu, 2, 1, 64, tile, 0, 1, 0, cap, sl,
                                 torch.float32, 4000, blocks=blocks)
    assert plan.info.max_item_tiles > 2100
    rows = torch.cat([torch.arange(n - 210, n, 9), torch.tensor([0, 63, 64, n - 1])]).cuda()
    key = torch.arange(n, device="cuda")
    dist = rows[:, None] - key
    keep = dist >= 0
    t = rows // tile
    keep &= ((key // tile == t[:, None]) | (t == count - 1)[:, None] | (t == count - 3)[:, None])
    ref = attend(q[rows], k, v, keep, dist, 0.125, cap, sl)
    check(o[rows], lse.t()[rows], ref, torch.float32, f"long lists {score}")


@pytest.mark.parametrize("kind", ["triangle", "causal", "blocksparse"])
@pytest.mark.parametrize("word,value", [(8, 9), (4, -1), (5, -1)])  # mode, first and last k-tile
def test_an_item_that_does_not_fit_shows_in_its_rows(kind, word, value):
    """One item's words out of range: the rows that it names are NaN, in the
    row normaliser too."""
    cu = [0, 70, 600, 1100]
    blocks, _ = _lists(cu, 64, 3)
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, 64, 2))
    plan = B.Plan(kind, cu, 8, 100, 70, 64, 4, 64, 2, blocks=blocks)
    words = plan.sched.tolist()
    for item in (0, plan.info.n_items // 2, plan.info.n_items - 1):
        at = 16 + 12 * item
        lo, hi = words[at] + words[at + 2], words[at] + words[at + 3]
        plan.sched[at + word] = value
        o = torch.zeros(q.shape, device="cuda")
        lse = torch.zeros(4, cu[-1], device="cuda")
        plan.run(q, k, v, o, lse, softcap=5.0)
        assert bool(torch.isnan(o[lo:hi]).all()), item
        assert bool(torch.isnan(lse[:, lo:hi]).all()), item
        plan.sched[at + word] = words[at + word]


@pytest.mark.parametrize("word,value", [(1, -5), (3, 10 ** 6), (4, -1)])  # r0, splits, partials
def test_a_merge_item_that_does_not_fit_shows_in_its_rows(word, value):
    cu = [0, 70, 600, 1100]
    q, k, v = (t.cuda() for t in draw_qkv(cu, 4, 1, 64, 2))
    plan = B.Plan("triangle", cu, 8, 100, 70, 64, 4, 64, 2)
    words = plan.sched.tolist()
    at = 16 + 12 * plan.info.n_items + 8 * (plan.info.n_merge_items - 1)
    lo, hi = words[at] + words[at + 1], words[at] + words[at + 2]
    plan.sched[at + word] = value
    o = torch.zeros(q.shape, device="cuda")
    lse = torch.zeros(4, cu[-1], device="cuda")
    plan.run(q, k, v, o, lse, softcap=5.0)
    if word != 1:  # (a row that is none names no rows)
        assert bool(torch.isnan(o[lo:hi]).all()) and bool(torch.isnan(lse[:, lo:hi]).all())
    assert bool(torch.isnan(o).any()) and bool(torch.isnan(lse).any())


@pytest.mark.parametrize("cap", [0.5, 30.0, 1024.0])
def test_error_of_a_cap(cap):
    """Rows of one key each, whose log-sum-exp is the capped score: products
    from far below to far past the cap, both signs.  With u = 2^-24, relative
    to the cap and in the order of the arithmetic: 1.5 u from the exponent's
    factor (3.3 u of it, times t (1 - tanh^2 t) <= 0.448), 1 u and 2 u from the
    exponential (an ulp of it) and its sum with one, 2 u from the reciprocal (an
    ulp), 1.2 u from the cap's factor, 2 u from the difference to a reference:
    9.7 u; the log-sum-exp adds 2.3 u of itself (two products, a constant)."""
    n, hq, d = 4000, 8, 64
    g = torch.Generator().manual_seed(28)
    q = torch.zeros(n, hq, d, dtype=torch.bfloat16)
    k = torch.zeros(n, 1, d, dtype=torch.bfloat16)
    size = torch.exp2(12.0 * torch.rand(n, generator=g) - 8.0) * cap  # |x|: cap 2^-8 .. 2^4
    k[:, 0, 0] = (8.0 * size * torch.sign(torch.randn(n, generator=g))).bfloat16()
    q[:, :, 0] = (1.0 + torch.rand(n, hq, generator=g)).bfloat16()
    q, k = q.cuda(), k.cuda()
    v = torch.zeros_like(k)
    plan = B.Plan("causal", list(range(n + 1)), 0, 1, 0, 64, hq, d)
    o, lse = torch.empty(n, hq, d, device="cuda"), torch.empty(hq, n, device="cuda")
    plan.run(q, k, v, o, lse, softmax_scale=0.125, softcap=cap)
    x = 0.125 * q[:, :, 0].double() * k[:, :, 0].double()  # [n, hq]
    err = (lse.t().double() - cap * torch.tanh(x / cap)).abs().max().item() / cap
    print(f"cap {cap}: {err * 2 ** 24:.2f} 2^-24")
    assert err <= 2.0 ** -20


def test_many_short_sequences_with_last_rows():
    """More q-tiles to join than a launch has rows of workgroups: 70000 packed
    sequences of one to three tokens, all of them Last rows."""
    lens = [1 + i % 3 for i in range(70000)]
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    g = torch.Generator().manual_seed(29)
    q = torch.randn(cu[-1], 32, 64, generator=g).bfloat16().cuda()
    k = torch.randn(cu[-1], 8, 64, generator=g).bfloat16().cuda()
    v = torch.randn(cu[-1], 8, 64, generator=g).bfloat16().cuda()
    args = (32, 8, 64, 128, 8, 64, 128, 20.0, None, torch.float32)
    o, lse = _run("triangle", cu, *args, qkv=(q, k, v))[3:5]
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all())
    for a, b in ((0, 40), (33000, 33040), (65530, 65545), (69950, 70000)):
        t0, t1 = cu[a], cu[b]
        part = [x - t0 for x in cu[a:b + 1]]
        out = _run("triangle", part, *args, qkv=(q[t0:t1], k[t0:t1], v[t0:t1]))
        assert torch.equal(out[3], o[t0:t1]) and torch.equal(out[4], lse[:, t0:t1])
        _verify("triangle", part, *out[:5], 128, 8, 64, 128, 20.0, None, f"sequences {a}..{b}")
