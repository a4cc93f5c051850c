"""GPU tests of attention over the 8-bit paged cache: what each of its forms (row
tiles of 16, 32, 128 and 256 rows) has to keep alike."""
import pytest
import torch

from tests.cache8_ref import Cache8
from tests.serving_ref import check
from tests.test_gpu_paged8 import _call

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
