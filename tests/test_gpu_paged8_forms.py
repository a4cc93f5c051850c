"""GPU tests of attention over the 8-bit paged cache: what each of its forms (row
tiles of 16, 32, 128 and 256 rows) has to keep alike."""
import math

import pytest
import torch

from tests.cache8_ref import Cache8
from tests.serving_ref import check, geometric_slopes
from tests.test_gpu_paged8 import _call, _q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("byte", [127, 246, 247])
@pytest.mark.parametrize("d,ql", [(64, 1), (128, 1), (64, 3), (128, 3), (64, 50), (128, 50),
                                  (128, 129)])  # 16, 32, 128 and 256 rows
def test_the_largest_scale_under_the_largest_weight(d, ql, byte):
    """A key whose probability against the row's reference, that of earlier
    keys, is just under the 2^8 from which on a row takes a new one, and rounds to
    2^8 in bf16; its value has the largest scale that the write makes, 2^120, and
    elements of 0 and 2^-6: no weight may become infinite."""
    heads, batch, n = 128, 16, 129  # many row tiles a share: few are cut
    c = Cache8([n], heads, d, 16, seed=41, sink=1.0)
    c.lens, c.table = [n] * batch, c.table.repeat(batch, 1)
    c.kv_lens = c.kv_lens.repeat(batch)
    c.k8.zero_()
    c.ks.fill_(127)
    c.k = torch.zeros_like(c.k)
    page = int(c.table[0, 8])
    c.k8[page, :, 0, :2] = 0x38  # 1
    c.k[page, :, 0, :2] = 1.0
    c.v8[page, :, 0, :] = 0x08  # 2^-6
    c.v8[page, :, 0, 5] = 0
    c.vs[page, :, 0] = byte
    c.v[page, :, 0, :] = 2.0 ** (byte - 127 - 6)
    c.v[page, :, 0, 5] = 0.0
    # the last key's score: 7.9985 ln 2 (2^7.9985 = 255.73), as a sum of two bf16
    # numbers, to 2^-17 of it; the others' 0
    want = 7.9985 * 0.6931471805599453 * d ** 0.5
    hi = torch.tensor(want).bfloat16().double()
    q = torch.zeros(batch * ql, heads, d)
    q[..., 0], q[..., 1] = float(hi), want - float(hi)
    q = q.bfloat16().cuda()
    o, l = _call(c, q, [ql] * batch, torch.float32, ragged=ql > 1)
    some = [0, 77, 127]
    c.k, c.v = c.k[:, some], c.v[:, some]
    check(o[:, some], l[:, some], c.reference(q[:, some], [ql] * batch, d ** -0.5), torch.float32,
          f"byte {byte} d {d} rows {ql}")


@pytest.mark.parametrize("d,lens,ql,hq,hkv", [
    (64, [100, 0, 70], [300, 200, 70], 4, 2),    # 128 rows
    (128, [20, 0, 33], [50, 30, 33], 4, 2),      # 128 rows
    (128, [100, 0, 70], [300, 200, 70], 4, 2),   # 256 rows
    (128, [700, 130, 1], [900, 129, 400], 7, 1)])
@pytest.mark.parametrize("prefix", [0, 77])
@pytest.mark.parametrize("score", ["plain", "cap", "slopes", "both"])
def test_rows_before_the_first_key_in_large_tiles(d, lens, ql, hq, hkv, prefix, score):
    """More query rows than keys: rows without any, and whole row tiles of them."""
    c = Cache8(lens, hkv, d, 16, prefix, seed=42)
    q = _q(sum(ql), hq, d, 42)
    cap = 20.0 if score in ("cap", "both") else None
    sl = geometric_slopes(hq) if score in ("slopes", "both") else None
    o, l = _call(c, q, ql, torch.float32, cap, sl, ragged=True)
    check(o, l, c.reference(q, ql, d ** -0.5, cap, sl), torch.float32, f"{d} {ql} {score}")
    none = max(0, ql[0] - lens[0])
    assert bool((o[:none] == 0).all()) and bool((l[:none] == -math.inf).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ql", [1, 4, 40, 150])  # 16, 32, 128 and (d = 128) 256 rows
@pytest.mark.parametrize("prefix", [0, 50])
def test_bad_pages_and_lengths_in_every_form(d, ql, prefix):
    """A page id outside the cache and a length past the table give NaN in the
    rows that need them, bit for bit nothing in the others; an entry behind
    the last key is not read."""
    lens = [200, 190, 180]
    c = Cache8(lens, 2, d, 16, prefix, seed=43)
    q = _q(3 * ql, 4, d, 43)
    good, gl = _call(c, q, [ql] * 3, torch.float32, ragged=ql > 1)
    check(good, gl, c.reference(q, [ql] * 3, d ** -0.5), torch.float32, f"{d} {ql} {prefix}")
    rows = [torch.arange(b * ql, (b + 1) * ql, device="cuda") for b in range(3)]
    table, kv = c.table.clone(), c.kv_lens.clone()

    def others_stand(b):
        rest = torch.cat([rows[i] for i in range(3) if i != b])
        assert torch.equal(o[rest], good[rest]) and torch.equal(l[rest], gl[rest])

    for page in (-1, c.k.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.table[1, 3] = page  # keys 48 .. 63
        o, l = _call(c, q, [ql] * 3, torch.float32, ragged=ql > 1)
        needs = torch.arange(190 - ql, 190, device="cuda") >= 48
        assert bool(o[rows[1][needs]].isnan().all()) and bool(l[rows[1][needs]].isnan().all())
        early = rows[1][~needs]
        assert torch.equal(o[early], good[early]) and torch.equal(l[early], gl[early])
        others_stand(1)
        c.table.copy_(table)
    c.table[1, 12] = -5
    o, l = _call(c, q, [ql] * 3, torch.float32, ragged=ql > 1)
    assert torch.equal(o, good) and torch.equal(l, gl)
    c.table.copy_(table)
    for n in (c.table.shape[1] * 16 + 1, 2 ** 31 - 1):
        c.kv_lens[2] = n
        o, l = _call(c, q, [ql] * 3, torch.float32, ragged=ql > 1)
        assert bool(o[rows[2]].isnan().all()) and bool(l[rows[2]].isnan().all())
        others_stand(2)
        c.kv_lens.copy_(kv)
    c.kv_lens[2] = -4  # no keys
    o, l = _call(c, q, [ql] * 3, torch.float32, ragged=ql > 1)
    assert bool((o[rows[2]] == 0).all()) and bool((l[rows[2]] == -math.inf).all())
    others_stand(2)
    c.kv_lens.copy_(kv)
    if prefix:
        keep = c.prefix_pages.clone()
        c.prefix_pages[2] = c.k.shape[0]
        o, l = _call(c, q, [ql] * 3, torch.float32, ragged=ql > 1)
        assert bool(o.isnan().all()) and bool(l.isnan().all())
        c.prefix_pages.copy_(keep)


@pytest.mark.parametrize("d,batch,ql,hq,hkv", [
    (64, 100, 4, 8, 2), (64, 480, 1, 8, 2), (64, 1024, 3, 2, 2), (128, 340, 4, 8, 2)])
@pytest.mark.parametrize("prefix", [0, 33])
def test_batches_whose_tables_take_workgroups_off_a_cu(d, batch, ql, hq, hkv, prefix):
    lens = [ql + (11 * i) % 300 for i in range(batch)]
    c = Cache8(lens, hkv, d, 64, prefix, seed=44)
    q = _q(batch * ql, hq, d, 44)
    o, l = _call(c, q, [ql] * batch, torch.float32, ragged=ql > 1)
    some = list(range(0, batch, 29)) + [batch - 1]
    at = torch.cat([torch.arange(i * ql, (i + 1) * ql) for i in some]).cuda()
    c.lens, c.table = [lens[i] for i in some], c.table[some]
    check(o[at], l[at], c.reference(q[at], [ql] * len(some), d ** -0.5), torch.float32,
          f"{d} {batch} {ql} {prefix}")
    assert bool(torch.isfinite(o).all())
