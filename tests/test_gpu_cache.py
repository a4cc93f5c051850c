"""GPU tests of page maps, cache writes, and a serving step of all operators."""
import random

import pytest
import torch

from paper_2507_21526_amd import binding as B
from paper_2507_21526_amd.inputs import draw_qkv
from tests.serving_ref import attend, check, geometric_slopes, page_map_ref

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _map(cached, new, table, free, n_free, page, count):
    b = len(cached)
    t = _ints(table).reshape(b, -1)
    kv, cu = _ints([9] * b), _ints([9] * (b + 1))
    slots, state = _ints([9] * count), _ints([9, 9])
    B.page_map(_ints(cached), _ints(new), t, _ints(free), _ints([n_free]), page, kv, cu, slots,
               state)
    return t.tolist(), kv.tolist(), cu.tolist(), slots.tolist(), state.tolist()


def _compare(cached, new, table, free, n_free, page, count):
    want = page_map_ref(cached, new, table, free, n_free, page, count)
    got = _map(cached, new, table, free, n_free, page, count)
    for g, w, name in zip(got, want, ("table", "kv_lens", "cu_new", "slots", "state")):
        assert g == w, name


def _setup(cached, page, width, rng, n_free):
    ids = rng.sample(range(4000), 4000)
    table = []
    for c in cached:
        n = -(-c // page)
        table.append([ids.pop() for _ in range(n)] + [-1] * (width - n))
    return table, [ids.pop() for _ in range(n_free)]


@pytest.mark.parametrize("seed", range(12))
def test_page_map(seed):
    rng = random.Random(seed)
    page = rng.choice([16, 32, 64, 128, 256])
    b = rng.choice([1, 2, 7, 63, 64, 65, 200, 256, 257])
    cached = [rng.choice([0, 1, page - 1, page, page + 1, rng.randrange(5 * page)])
              for _ in range(b)]
    new = [rng.choice([0, 1, 1, page, rng.randrange(3 * page)]) for _ in range(b)]
    need = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(cached, new))
    table, free = _setup(cached, page, 9, rng, need + 5)
    _compare(cached, new, table, free, need + rng.choice([0, 1, 5]), page,
             sum(new) + rng.choice([0, 1, 1500]))


def test_page_map_sizes():
    rng = random.Random(5)
    # the largest batch, one token each; a long prompt over many workgroups
    cached = [rng.randrange(40) for _ in range(1024)]
    table, free = _setup(cached, 16, 4, rng, 500)
    _compare(cached, [1] * 1024, table, free, 480, 16, 1024)
    _compare([0], [9000], [[-1] * 600], list(range(700)), 650, 16, 9000)
    _compare([0, 0], [0, 0], [[-1], [-1]], [3], 1, 16, 3)
    _compare([5], [0], [[7]], [3], 1, 16, 0)


def test_page_map_without_requests():
    t = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    kv, cu, slots, state = _ints([]), _ints([9]), _ints([9] * 4), _ints([9, 9])
    B.page_map(_ints([]), _ints([]), t, _ints([1, 2]), _ints([2]), 16, kv, cu, slots, state)
    assert cu.tolist() == [0] and slots.tolist() == [-1] * 4 and state.tolist() == [2, 0]


@pytest.mark.parametrize("cached,new,width,n_free,count,bits", [
    ([10, 20], [7, 30], 6, 2, 37, B.MAP_NO_PAGES),
    ([10, 20], [7, 30], 3, 9, 37, B.MAP_TABLE_WIDTH),
    ([10, -1], [7, 30], 6, 9, 37, B.MAP_BAD_LENGTH),
    ([10, 20], [-7, 30], 6, 9, 37, B.MAP_BAD_LENGTH),
    ([10, 20], [7, 30], 6, 9, 36, B.MAP_SLOT_COUNT),
    ([10, 20], [7, 30], 6, 11, 37, B.MAP_BAD_FREE),
    ([10, 20], [7, 30], 6, -1, 37, B.MAP_BAD_FREE | B.MAP_NO_PAGES),
    ([10, 2 ** 31 - 1], [7, 2 ** 31 - 1], 6, 1, 3,
     B.MAP_NO_PAGES | B.MAP_TABLE_WIDTH | B.MAP_SLOT_COUNT),
])
def test_page_map_is_all_or_nothing(cached, new, width, n_free, count, bits):
    table = [[40] + [-1] * (width - 1), [41, 42] + [-1] * (width - 2)]
    free = list(range(10))
    got = _map(cached, new, table, free, n_free, 16, count)
    assert got == (table, cached, [0, 0, 0], [-1] * count, [n_free, bits])
    assert got == tuple(page_map_ref(cached, new, table, free, n_free, 16, count))


def test_page_map_of_entries_that_are_no_pages():
    """A token in an old page whose entry is none gets no slot."""
    got = _map([20, 3], [2, 2], [[5, -1], [2 ** 31 - 1, -1]], [7], 1, 16, 4)
    assert got[3] == [-1] * 4 and got[4] == [1, 0]


@pytest.mark.parametrize("tokens,hkv,d,page,fused", [
    (1, 1, 64, 16, False), (7, 3, 128, 16, True), (333, 8, 128, 64, True), (64, 2, 64, 256, False),
    (1000, 5, 64, 32, True)])
def test_cache_write(tokens, hkv, d, page, fused):
    g = torch.Generator().manual_seed(tokens)
    if fused:  # views of a projection's output, other strides for k and v
        x = torch.randn(tokens, 2 * hkv + 3, d, generator=g).bfloat16().cuda()
        k = x[:, 3:3 + hkv]
        v = torch.randn(hkv, tokens, d, generator=g).bfloat16().cuda().transpose(0, 1)
    else:
        k = torch.randn(tokens, hkv, d, generator=g).bfloat16().cuda()
        v = torch.randn(tokens, hkv, d, generator=g).bfloat16().cuda()
    pages = tokens // page + 4
    kc = torch.randn(pages, hkv, page, d, generator=g).bfloat16().cuda()
    vc = torch.randn(pages, hkv, page, d, generator=g).bfloat16().cuda()
    slots = torch.randperm(pages * page, generator=g)[:tokens].to(torch.int32)
    if tokens > 3:
        slots[1], slots[2] = -1, pages * page  # skipped
    wk, wv = kc.clone(), vc.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            wk[s // page, :, s % page], wv[s // page, :, s % page] = k[t], v[t]
    B.kv_cache_write(k, v, slots.cuda(), kc, vc)
    torch.cuda.synchronize()
    assert torch.equal(kc, wk) and torch.equal(vc, wv)


def test_cache_write_of_one_row_and_head():
    """Dimensions of one may have any stride."""
    x = torch.randn(40 * 64, device="cuda").bfloat16()
    k, v = x.as_strided((1, 1, 64), (3, 5, 1)), x.as_strided((1, 1, 64), (1, 1, 1), 64)
    kc = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    B.kv_cache_write(k, v, _ints([20]), kc, vc)
    assert torch.equal(kc[1, 0, 4], x[:64]) and torch.equal(vc[1, 0, 4], x[64:128])


def test_cache_write_keeps_bits():
    """Rows are moved as they are: NaN payloads, infinities, denormals."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    k = bits.reshape(1024, 1, 64).cuda()
    v = bits.flip(0).reshape(1024, 1, 64).cuda()
    kc = torch.zeros(64, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    B.kv_cache_write(k, v, torch.arange(1024, dtype=torch.int32, device="cuda"), kc, vc)
    assert torch.equal(kc.view(torch.int16).flatten(), k.view(torch.int16).flatten())
    assert torch.equal(vc.view(torch.int16).flatten(), v.view(torch.int16).flatten())


@pytest.mark.parametrize("score", ["plain", "both"])
def test_a_serving_run(score):
    """Prompts through the prefill pass and into the cache, then decoded
    tokens through a captured step of map, write and attention: every row is
    that of attention over the whole sequence."""
    hq, hkv, d, page, steps = 8, 2, 128, 16, 4
    lens = [130, 17, 64]
    b, width = 3, 12
    cap, sl = (25.0, geometric_slopes(hq)) if score == "both" else (None, None)
    seqs = [[t.cuda() for t in draw_qkv([0, n + steps], hq, hkv, d, 50 + n)] for n in lens]
    # prefill
    cu = [0, 130, 147, 211]
    q, k, v = (torch.cat([s[i][:n] for s, n in zip(seqs, lens)]) for i in range(3))
    o = torch.empty_like(q)
    B.Plan("causal", cu, 0, 1, 0, 64, hq, d).run(q, k, v, o, softcap=cap, slopes=sl)
    kc = torch.full((40, hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    vc = kc.clone()
    table = torch.full((b, width), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.randperm(40, device="cuda").to(torch.int32), _ints([40])
    cached, kv, cu_new = _ints([0, 0, 0]), _ints([0] * 3), _ints([0] * 4)
    slots, state = _ints([0] * 211), _ints([0, 0])
    B.page_map(cached, _ints(lens), table, free, n_free, page, kv, cu_new, slots, state)
    B.kv_cache_write(k, v, slots, kc, vc)
    # one decode step, captured
    one, nk = _ints([1, 1, 1]), torch.zeros(b, hkv, d, dtype=torch.bfloat16, device="cuda")
    nq, nv = torch.zeros(b, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(nk)
    no, nlse = torch.zeros_like(nq), torch.zeros(hq, b, device="cuda")
    slot1 = _ints([0] * 3)
    plan = B.PagedPlan(b, b, hq, hkv, d)

    def step():
        cached.copy_(kv)
        n_free.copy_(state[:1])
        B.page_map(cached, one, table, free, n_free, page, kv, cu_new, slot1, state)
        B.kv_cache_write(nk, nv, slot1, kc, vc)
        plan.run(nq, kc, vc, no, kv, table, lse=nlse, softcap=cap, slopes=sl)

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
            ref = attend(seqs[i][0][m - 1:m], seqs[i][1][:m], seqs[i][2][:m], dist >= 0, dist,
                         d ** -0.5, cap, sl)
            check(no[i:i + 1], nlse.t()[i:i + 1], ref, torch.bfloat16, f"step {t} request {i}")
    for i, n in enumerate(lens):
        dist = torch.arange(n, device="cuda")[:, None] - torch.arange(n, device="cuda")
        ref = attend(seqs[i][0][:n], seqs[i][1][:n], seqs[i][2][:n], dist >= 0, dist, d ** -0.5,
                     cap, sl)
        check(o[cu[i]:cu[i + 1]], None, ref, torch.bfloat16, f"prompt {i}")


def test_cache_write_of_more_rows_than_threads():
    """2^28 rows and more, 2^32 chunks: one row's views repeated (strides of
    zero), a few of them with a slot."""
    n, hkv, d = (1 << 25) + 5, 8, 128
    k = torch.randn(1, hkv, d, device="cuda").bfloat16()
    v = torch.randn(1, hkv, d, device="cuda").bfloat16()
    kc = torch.zeros(2, hkv, 16, d, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    slots = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 1, 1 << 24, n - 6, n - 1], device="cuda")
    slots[at] = torch.arange(3, 8, dtype=torch.int32, device="cuda")
    B.kv_cache_write(k.expand(n, hkv, d), v.expand(n, hkv, d), slots, kc, vc)
    assert torch.equal(kc[0, :, 3:8], k[0][:, None].expand(hkv, 5, d))
    assert torch.equal(vc[0, :, 3:8], v[0][:, None].expand(hkv, 5, d))
    assert not bool(kc[0, :, :3].any()) and not bool(kc[0, :, 8:].any()) and not bool(kc[1].any())
