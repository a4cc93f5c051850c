"""Host tests of how 8-bit paged attention cuts its work: as many shares as
workgroups fit the chip with their tables of lengths, or a whole number of times
as many, so that it is never some of them that start when the others end."""
import pytest

from paper_2507_21526_amd import binding as B

CUS, LDS, GRANULE = 256, 160 * 1024, 1280


def shares_of_a_cu(batch, tokens, ragged, hq, hkv, d, rows):
    """Of the layout: two pieces of `rows` rows a
    share and kv head in the workspace (d values and a log-sum-exp each), beside
    32 bytes a row tile."""
    size = B.ta_paged_q8_workspace_bytes(batch, tokens, ragged, False, hq, hkv, d)
    tiles = batch + (tokens * (hq // hkv) // rows if ragged else 0)
    shares = (size - 32 * tiles) // (2 * hkv * rows * (d + 1) * 4)
    return shares * hkv / CUS


def fit(batch, tokens, ragged, hq, hkv, d, rows):
    """What LDS holds: two waves with two stages of 64 keys, K and V, and 512
    bytes of scales, the next query rows, 556 bytes beside; and the tables: a word a
    row tile (and one), one a request, with query offsets two more (and one each)."""
    own = 2 * 2 * (2 * 64 * d + 512) + rows * 2 * d + 556
    tiles = batch + (tokens * (hq // hkv) // rows if ragged else 0)
    tables = 4 * (tiles + 1 + batch + (2 * (batch + 1) if ragged else 0))
    return min(2 if d == 128 else 4, LDS // (-(-(own + tables) // GRANULE) * GRANULE))


@pytest.mark.parametrize("d,batch,tokens,hq,hkv,want", [
    (128, 300, 4, 32, 8, 2), (128, 400, 4, 32, 8, 1), (128, 1024, 4, 16, 2, 1),
    (64, 80, 4, 32, 8, 4), (64, 100, 4, 32, 8, 3), (64, 300, 4, 32, 8, 3), (64, 1024, 3, 8, 8, 2),
    (64, 440, 1, 32, 8, 4), (64, 480, 1, 32, 8, 3), (64, 1024, 1, 32, 8, 3),
    (128, 1024, 1, 32, 8, 2), (128, 1, 1, 32, 8, 2), (64, 1, 1, 8, 1, 4)])
def test_shares_come_in_whole_rounds(d, batch, tokens, hq, hkv, want):
    ragged = tokens > 1
    case = (batch, batch * tokens, ragged, hq, hkv, d, 32 if ragged else 16)
    assert fit(*case) == want
    most = 2 if d == 128 else 4
    assert shares_of_a_cu(*case) == most // want * want


def test_bf16_shares_stand():
    for d, per_cu in ((128, 2), (64, 4)):
        for batch in (80, 400, 1024):
            size = B.ta_paged_workspace_bytes(batch, 4 * batch, True, False, 32, 8, d)
            assert size // (2 * 8 * 32 * (d + 1) * 4) * 8 // CUS == per_cu
