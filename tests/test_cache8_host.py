"""The 8-bit cache's refusals and its plain forms: no GPU needed; every call
here is rejected by the host before any HIP call."""
import ctypes
import re

import pytest
import torch

from paper_2507_21526_amd import binding as B
from tests.cache8_ref import E4M3, quantise, values

P = ctypes.c_void_p
M = 1 << 20  # bytes between arguments, none of which is dereferenced


def test_plain_quantisation():
    """The search agrees with torch's conversion of rows in range, and with
    hand-made rows at the borders of a scale."""
    assert len(E4M3) == 127 and E4M3[1] == 2.0 ** -9 and E4M3[126] == 448.0
    g = torch.Generator().manual_seed(1)
    x = torch.randn(500, 64, generator=g).bfloat16()
    codes, scales = quantise(x)
    e = scales.int() - 127
    want = torch.ldexp(x.float(), -e[:, None]).to(torch.float8_e4m3fn)
    assert torch.equal(codes.view(torch.float8_e4m3fn).float(), want.float())
    # half a step, 2^-4 of a value, or of the least normal element
    err = (values(codes, scales) - x.double()).abs()
    tol = torch.maximum(x.double().abs(), torch.exp2(e.double() - 6)[:, None]) * 2.0 ** -4
    assert bool((err <= tol).all())
    top = torch.tensor([0.0, 448.0, 450.0, 1.75, 1.7578125, 2.0 ** -130, 2.0 ** -91, 3.3895e38,
                        2.0 ** 127])
    rows = torch.stack([top, torch.zeros(9)], 1).bfloat16()
    codes, scales = quantise(rows)
    assert (scales.int() - 127).tolist() == [-100, 0, 1, -8, -7, -100, -99, 120, 119]
    assert values(codes, scales)[:, 0].tolist() == [
        0.0, 448.0, 448.0, 1.75, 1.75, 0.0, 2.0 ** -91, 240 * 2.0 ** 120, 2.0 ** 127]
    rows = torch.tensor([[1.0, float("inf"), float("nan"), -float("inf")]]).bfloat16()
    codes, scales = quantise(rows)
    assert codes[0, 1:].tolist() == [127, 127, 255] or bool(
        torch.isnan(values(codes, scales)[0, 1:]).all())
    assert scales.tolist() == [127 - 8]


def _write(k=M, v=2 * M, ks=128, kh=64, slots=3 * M, tokens=4, kc=4 * M, ksc=5 * M, vc=6 * M,
           vsc=7 * M, pages=4, hkv=2, page=16, d=64):
    return B.lib().kv_cache_write_q8(P(k), P(v), ks, kh, 128, 64, P(slots), tokens, P(kc), P(ksc),
                                     P(vc), P(vsc), pages, hkv, page, d, None)


def test_write_refusals():
    inv, uns = B.TA_ERR_INVALID_ARG, B.TA_ERR_UNSUPPORTED
    for want, kw in [
            (inv, dict(tokens=-1)), (inv, dict(pages=-1)), (inv, dict(hkv=0)), (uns, dict(d=96)),
            (uns, dict(page=20)), (uns, dict(pages=1 << 28)), (inv, dict(k=0)), (inv, dict(v=0)),
            (inv, dict(slots=0)), (inv, dict(kc=0)), (inv, dict(ksc=0)), (inv, dict(vsc=0)),
            (inv, dict(k=M + 8)), (inv, dict(kc=4 * M + 2)), (inv, dict(ks=-128)),
            (inv, dict(ks=100)), (inv, dict(kh=4)),
            (inv, dict(ksc=4 * M + 8191)),       # the last byte of k_cache
            (inv, dict(vsc=5 * M + 127)),        # the last K scale
            (inv, dict(ksc=3 * M + 12)),         # the last slot
            (inv, dict(vc=M + 896 - 8192 + 16))]:  # up to k's last row
        assert _write(**kw) == want, (kw, B.ta_last_error())
    assert "overlap" in B.ta_last_error()
    assert "kv_cache_write_q8" in B.ta_last_error()
    assert _write(tokens=0) == B.TA_OK


def _read(q8=True, kc=M, ks=2 * M, vc=3 * M, vs=4 * M, table=5 * M, batch=2, width=4, cu=6 * M,
          starts=7 * M, k=8 * M, v=9 * M, kt=128, kh=64, vt=128, vh=64, total=6, pages=4, hkv=2,
          page=16, d=64):
    rest = (P(table), batch, width, P(cu), P(starts), P(k), P(v), kt, kh, vt, vh, total, pages,
            hkv, page, d, None)
    if q8:
        return B.lib().kv_cache_read_q8(P(kc), P(ks), P(vc), P(vs), *rest)
    return B.lib().kv_cache_read(P(kc), P(vc), *rest)


@pytest.mark.parametrize("q8", [False, True])
def test_read_refusals(q8):
    inv, uns = B.TA_ERR_INVALID_ARG, B.TA_ERR_UNSUPPORTED
    cases = [
        (inv, dict(batch=-1)), (inv, dict(width=-1)), (inv, dict(total=-1)), (inv, dict(pages=-1)),
        (inv, dict(hkv=0)), (uns, dict(batch=1025)), (uns, dict(d=32)), (uns, dict(page=8)),
        (uns, dict(pages=1 << 28)), (uns, dict(width=1 << 28)), (uns, dict(total=1 << 31)),
        (inv, dict(kc=0)), (inv, dict(vc=0)), (inv, dict(table=0)), (inv, dict(cu=0)),
        (inv, dict(k=0)), (inv, dict(v=0)), (inv, dict(k=8 * M + 8)), (inv, dict(vc=3 * M + 4)),
        (inv, dict(kt=100)), (inv, dict(kt=64)),  # tokens on the heads before
        (inv, dict(kt=-128)), (inv, dict(kh=0)), (inv, dict(vh=56)), (inv, dict(kt=0)),
        (inv, dict(v=8 * M)), (inv, dict(v=8 * M + 128)), (inv, dict(v=8 * M + 1408)),
        (inv, dict(k=M)), (inv, dict(v=5 * M - 1520)), (inv, dict(k=6 * M)), (inv, dict(v=7 * M))]
    if q8:
        cases += [(inv, dict(ks=0)), (inv, dict(vs=0)), (inv, dict(k=2 * M + 112))]
    for want, kw in cases:
        assert _read(q8, **kw) == want, (kw, B.ta_last_error())
    assert _read(q8, total=0) == B.TA_OK and _read(q8, batch=0) == B.TA_OK
    # k and v that alternate in one buffer pass these checks: what is refused
    # here is the table that lies on them
    for kw in (dict(v=8 * M + 2 * 128, kt=256, vt=256),              # [T, 2 hkv, d]
               dict(v=8 * M + 2 * 64, kt=256, vt=256, kh=128, vh=128),  # [T, hkv, 2, d]
               dict(v=8 * M + 2 * 64 * 6, kt=64, kh=768, vt=64, vh=768)):  # [hkv, 2, T, d]
        assert _read(q8, table=8 * M, **kw) == inv
        assert "an output overlaps another argument" in B.ta_last_error(), kw
    for kw in (dict(v=8 * M + 2 * 120, kt=256, vt=256),
               dict(v=8 * M + 2 * 136, kt=256, vt=256),  # its last head on the next token's k
               dict(v=8 * M + 2 * 128, kt=256, vt=384)):
        assert _read(q8, table=8 * M, **kw) == inv
        assert "rows of k or v overlap" in B.ta_last_error(), kw


def _paged(q=0, kc=M, ks=2 * M, vc=3 * M, vs=4 * M, o=5 * M, o_dtype=0, kv=6 * M, cu=7 * M,
           table=8 * M, batch=2, width=4, prefix=0, prefix_len=0, total=6, hq=8, hkv=2, d=64,
           pages=9, page=16, scale=0.1, cap=0.0, ws=16 * M, ws_bytes=1 << 40):
    return B.lib().paged_attn_fwd_q8(
        P(q or 12 * M), P(kc), P(ks), P(vc), P(vs), P(o), o_dtype, None, P(kv), P(cu), P(table),
        batch, width, P(prefix), prefix_len, total, hq, hkv, d, pages, page, scale, cap, None,
        P(ws), ws_bytes, None)


def test_paged_refusals():
    inv, uns = B.TA_ERR_INVALID_ARG, B.TA_ERR_UNSUPPORTED
    for want, kw in [
            (inv, dict(batch=-1)), (inv, dict(total=-1)), (inv, dict(width=-1)),
            (inv, dict(prefix_len=-1)), (inv, dict(pages=-1)), (inv, dict(pages=0)),
            (inv, dict(hq=0)), (inv, dict(hq=7)), (uns, dict(hq=18)), (uns, dict(d=80)),
            (uns, dict(page=48)), (inv, dict(o_dtype=2)), (inv, dict(scale=0.0)),
            (inv, dict(cap=-1.0)), (uns, dict(cap=1025.0)), (inv, dict(cu=0)),
            (uns, dict(batch=1025)), (uns, dict(width=1 << 28)), (uns, dict(pages=1 << 28)),
            (uns, dict(total=200000, batch=600)), (inv, dict(kc=0)), (inv, dict(ks=0)),
            (inv, dict(vs=0)), (inv, dict(kv=0)), (inv, dict(table=0)), (inv, dict(prefix_len=5)),
            (inv, dict(q=12 * M + 4)), (inv, dict(kc=M + 8)), (inv, dict(ks=2 * M + 2)),
            (inv, dict(vs=4 * M + 1)), (B.TA_ERR_WORKSPACE, dict(ws=0)),
            (B.TA_ERR_WORKSPACE, dict(ws_bytes=100)), (B.TA_ERR_WORKSPACE, dict(ws=16 * M + 4)),
            (inv, dict(o=12 * M)), (inv, dict(o=M)), (inv, dict(o=2 * M)), (inv, dict(o=4 * M + 272)),
            (inv, dict(ks=16 * M + 64))]:
        assert _paged(**kw) == want, (kw, B.ta_last_error())
    assert "paged_attn_fwd_q8" in B.ta_last_error()
    assert _paged(batch=0, total=0) == B.TA_OK


def test_workspace_bytes():
    f = B.ta_paged_q8_workspace_bytes
    assert f(4, 4, False, False, 8, 2, 128) > 0
    assert f(4, 4, False, True, 8, 2, 128) > f(4, 4, False, False, 8, 2, 128)
    for bad in ((-1, 4, False, False, 8, 2, 128), (4, -1, False, False, 8, 2, 128),
                (4, 4, False, False, 7, 2, 128), (4, 4, False, False, 8, 2, 96)):
        assert f(*bad) == 0


def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _b(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _c(*shape):
    return torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn)


def _s(*shape):
    return torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e8m0fnu)


def test_binding_refuses_tensors_that_do_not_fit():
    """Host tensors: the last check of each call is that they are on a GPU."""
    caches = dict(k_cache=_c(3, 2, 16, 64), v_cache=_c(3, 2, 16, 64), k_scale=_s(3, 2, 16),
                  v_scale=_s(3, 2, 16))
    wrong = [("k_cache", _b(3, 2, 16, 64), "k_cache must be torch.float8_e4m3fn"),
             ("v_cache", _c(3, 2, 32, 64), "v_cache"), ("k_scale", None, "k_scale"),
             ("v_scale", None, "v_scale"), ("k_scale", _s(3, 2, 32), "k_scale must be (3, 2, 16)"),
             ("v_scale", _s(3, 2, 16).view(torch.uint8), "v_scale must be torch.float8_e8m0fnu"),
             ("k_scale", _s(3, 16, 2).transpose(1, 2), "contiguous"),
             ("k_cache", _c(3, 2, 64), "k_cache must be a tensor")]
    ok = dict(k=_b(5, 2, 64), v=_b(5, 2, 64), slots=_i(5), **caches)
    for name, value, msg in wrong + [
            ("k", _b(5, 2, 64).float(), "k must be a bfloat16"), ("slots", _i(4), "slots must be"),
            ("slots", _i(5), "must be on a GPU")]:
        with pytest.raises(ValueError, match=re.escape(msg)):
            B.kv_cache_write(**{**ok, name: value})
    ok = dict(k=_b(5, 2, 64), v=_b(5, 2, 64), block_table=_i(3, 2), cu=_i(4), starts=_i(3),
              **caches)
    for name, value, msg in wrong + [
            ("v", _b(4, 2, 64), "differ"), ("cu", _i(3), "starts must be"),
            ("cu", _i(0), "cu must be a tensor"), ("cu", _i(4, 1), "cu must be a tensor"),
            ("starts", _i(2), "starts must be"), ("block_table", _i(2, 2), "block_table"),
            ("k", _b(5, 3, 64), "differ"), ("cu", _i(4).long(), "cu must be torch.int32"),
            ("starts", None, "must be on a GPU")]:
        with pytest.raises(ValueError, match=re.escape(msg)):
            B.kv_cache_read(**{**ok, name: value})
    with pytest.raises(ValueError, match="k_cache must be torch.bfloat16"):
        B.kv_cache_read(**{**ok, "k_scale": None, "v_scale": None})
    ok = dict(q=_b(3, 4, 64), o=_b(3, 4, 64), lse=torch.zeros(4, 3), kv_lens=_i(3), cu_q=None,
              block_table=_i(3, 2), prefix_pages=None, prefix_len=0, softmax_scale=0.1,
              softcap=None, slopes=None, workspace=None, **caches)
    for name, value, msg in wrong + [("lse", None, "must be on a GPU")]:
        with pytest.raises(ValueError, match=re.escape(msg)):
            B.paged_attn_fwd(**{**ok, name: value})
