"""The serving operators' refusals: every call here is rejected by the host,
before any HIP call (no GPU needed)."""
import ctypes
import re

import pytest
import torch

from paper_2507_21526_amd import binding as B

FAKE = 0x10000  # never dereferenced: every call below fails its checks first
P = ctypes.c_void_p


def _map(batch=2, page=16, width=4, capacity=8, slots=10, cached=FAKE, kv=FAKE + 4096,
         n_free=FAKE + 8192, state=FAKE + 12288, table=FAKE + 16384):
    return B.lib().ta_page_map(P(cached), P(FAKE + 512), batch, page, P(table), width,
                               P(FAKE + 20480), capacity, P(n_free), P(kv), P(FAKE + 24576),
                               P(FAKE + 28672), slots, P(state), None)


def test_page_map_refusals():
    bad = {"batch": -1, "width": -1, "capacity": -1, "slots": -1}
    for name, value in bad.items():
        assert _map(**{name: value}) == B.TA_ERR_INVALID_ARG, name
    assert _map(batch=1025) == B.TA_ERR_UNSUPPORTED
    for page in (0, 8, 24, 512, -16):
        assert _map(page=page) == B.TA_ERR_UNSUPPORTED, page
    assert _map(width=1 << 28) == B.TA_ERR_UNSUPPORTED
    assert _map(slots=1 << 31) == B.TA_ERR_UNSUPPORTED
    for name in ("cached", "kv", "n_free", "state", "table"):
        assert _map(**{name: 0}) == B.TA_ERR_INVALID_ARG, name
    assert _map(kv=FAKE) == B.TA_ERR_INVALID_ARG  # an output on an input
    assert "overlap" in B.ta_last_error()
    assert _map(state=FAKE + 8192) == B.TA_ERR_INVALID_ARG
    assert _map(state=FAKE + 28672 + 36) == B.TA_ERR_INVALID_ARG  # on the last slot


def _write(k=FAKE, kc=FAKE + (1 << 20), ks=128, kh=64, tokens=4, pages=4, hkv=2, page=16, d=64, slots=FAKE):
    return B.lib().kv_cache_write(P(k), P(FAKE), ks, kh, 128, 64, P(slots), tokens, P(kc),
                                  P(FAKE + (1 << 21)), pages, hkv, page, d, None)


def test_cache_write_refusals():
    assert _write(tokens=-1) == B.TA_ERR_INVALID_ARG
    assert _write(pages=-1) == B.TA_ERR_INVALID_ARG
    assert _write(hkv=0) == B.TA_ERR_INVALID_ARG
    assert _write(d=96) == B.TA_ERR_UNSUPPORTED
    assert _write(page=20) == B.TA_ERR_UNSUPPORTED
    assert _write(pages=1 << 28) == B.TA_ERR_UNSUPPORTED
    assert _write(k=0) == B.TA_ERR_INVALID_ARG
    assert _write(slots=0) == B.TA_ERR_INVALID_ARG
    assert _write(k=FAKE + 8) == B.TA_ERR_INVALID_ARG
    assert _write(kc=FAKE + (1 << 20) + 2) == B.TA_ERR_INVALID_ARG
    assert _write(ks=-128) == B.TA_ERR_INVALID_ARG
    assert _write(k=FAKE + (1 << 20) - 896) == B.TA_ERR_INVALID_ARG  # its last row on the cache
    assert "overlap" in B.ta_last_error()
    assert _write(ks=100) == B.TA_ERR_INVALID_ARG
    assert _write(kh=4) == B.TA_ERR_INVALID_ARG
    assert _write(tokens=0) == B.TA_OK  # nothing to do, nothing launched


M = 1 << 20  # bytes between the paged call's arguments


def _paged(q=FAKE, o_dtype=0, kv=FAKE + 4 * M, cu=FAKE + 5 * M, table=FAKE + 6 * M, batch=2, width=4, prefix=0,
           prefix_len=0, total=6, hq=8, hkv=2, d=64, pages=9, page=16, scale=0.1, cap=0.0,
           ws=FAKE + 8 * M, ws_bytes=1 << 40, o=FAKE + 3 * M):
    return B.lib().paged_attn_fwd(P(q), P(FAKE + M), P(FAKE + 2 * M), P(o), o_dtype, None, P(kv), P(cu),
                                  P(table), batch, width, P(prefix), prefix_len, total, hq, hkv, d,
                                  pages, page, scale, cap, None, P(ws), ws_bytes, None)


def test_paged_refusals():
    inv, uns = B.TA_ERR_INVALID_ARG, B.TA_ERR_UNSUPPORTED
    for want, kw in [
            (inv, dict(batch=-1)), (inv, dict(total=-1)), (inv, dict(width=-1)),
            (inv, dict(prefix_len=-1)), (inv, dict(pages=-1)), (inv, dict(pages=0)),
            (inv, dict(hq=0)), (inv, dict(hkv=0)), (inv, dict(hq=7)), (uns, dict(hq=18)),
            (uns, dict(d=80)), (uns, dict(page=48)), (inv, dict(o_dtype=2)),
            (inv, dict(scale=0.0)), (inv, dict(scale=float("inf"))), (inv, dict(cap=-1.0)),
            (inv, dict(cap=float("nan"))), (uns, dict(cap=1025.0)), (inv, dict(cap=1e-41)),
            (inv, dict(cu=0)),                      # six rows for two requests
            (uns, dict(batch=1025)), (uns, dict(width=1 << 28)), (uns, dict(pages=1 << 28)),
            (uns, dict(total=1 << 30)), (uns, dict(total=200000, batch=600)),
            (inv, dict(q=0)), (inv, dict(kv=0)), (inv, dict(table=0)),
            (inv, dict(prefix_len=5)), (inv, dict(q=FAKE + 4)),
            (B.TA_ERR_WORKSPACE, dict(ws=0)), (B.TA_ERR_WORKSPACE, dict(ws_bytes=100)),
            (B.TA_ERR_WORKSPACE, dict(ws=FAKE + 8 * M + 4)),
            (inv, dict(o=FAKE)), (inv, dict(o=FAKE + M)), (inv, dict(kv=FAKE + 8 * M + 64)),
            (inv, dict(prefix=FAKE + 3 * M, prefix_len=1))]:
        assert _paged(**kw) == want, (kw, B.ta_last_error())
    assert _paged(batch=0, total=0) == B.TA_OK  # nothing to do


def test_paged_workspace_bytes():
    f = B.ta_paged_workspace_bytes
    assert f(4, 4, False, False, 8, 2, 128) > 0
    assert f(4, 4, False, True, 8, 2, 128) > f(4, 4, False, False, 8, 2, 128)
    for bad in ((-1, 4, False, False, 8, 2, 128), (4, -1, False, False, 8, 2, 128),
                (4, 4, False, False, 7, 2, 128), (4, 4, False, False, 8, 2, 96)):
        assert f(*bad) == 0


def _scored(kind="causal", cap=5.0, slopes=0, **kw):
    _, info = B.ta_build_schedule(kind, [0, 100], 4, 8, 2, 64)
    for name, value in kw.pop("info", {}).items():
        setattr(info, name, value)
    a = dict(q=FAKE, o_dtype=0, total=100, hq=8, hkv=2, d=64, scale=0.1, ws=FAKE,
             ws_bytes=1 << 40, sched=FAKE)
    a.update(kw)
    return B.lib().scored_attn_fwd(P(a["q"]), P(FAKE), P(FAKE), P(FAKE), a["o_dtype"], None,
                                   P(a["sched"]), ctypes.byref(info), a["total"], a["hq"],
                                   a["hkv"], a["d"], a["scale"], cap, P(slopes), P(a["ws"]),
                                   a["ws_bytes"], None)


def test_scored_refusals():
    inv, uns, mis = B.TA_ERR_INVALID_ARG, B.TA_ERR_UNSUPPORTED, B.TA_ERR_SCHEDULE_MISMATCH
    assert B.lib().scored_attn_fwd(*[None] * 4, 0, None, None, None, 100, 8, 2, 64, 0.1, 5.0,
                                   None, None, 0, None) == inv
    for want, kw in [
            (inv, dict(cap=0.0)),  # neither a cap nor slopes
            (inv, dict(cap=-2.0)), (inv, dict(cap=float("inf"))), (uns, dict(cap=2000.0)),
            (inv, dict(cap=1e-41)), (mis, dict(total=99)), (inv, dict(hq=7)),
            (uns, dict(hq=18)), (uns, dict(d=96)), (inv, dict(o_dtype=9)), (inv, dict(scale=-1.0)),
            (inv, dict(q=0)), (inv, dict(q=FAKE + 2)), (inv, dict(sched=0)),
            (uns, dict(hq=65536, hkv=8192, d=128)),
            (mis, dict(info=dict(version=1))), (mis, dict(info=dict(kind=5))),
            (uns, dict(info=dict(tile=32))), (mis, dict(info=dict(words=3))),
            (mis, dict(info=dict(n_items=-1)))]:
        assert _scored(**kw) == want, (kw, B.ta_last_error())
    assert _scored("triangle", ws=0) == B.TA_ERR_WORKSPACE
    assert _scored("triangle", ws_bytes=8) == B.TA_ERR_WORKSPACE
    assert _scored("triangle", ws=FAKE + 4) == inv


def _i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _b(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_binding_refuses_tensors_that_do_not_fit():
    """Host tensors: the last check of each call is that they are on a GPU."""
    ok = dict(cached_lens=_i(3), new_lens=_i(3), block_table=_i(3, 4), free_pages=_i(9),
              n_free=_i(1), page_size=16, kv_lens=_i(3), cu_new=_i(4), slots=_i(7), state=_i(2))
    for name, value, msg in [
            ("cached_lens", _i(3, 1), "cached_lens must be"), ("new_lens", _i(2), "new_lens"),
            ("block_table", _i(2, 4), "block_table"), ("block_table", _i(4, 3).t(), "contiguous"),
            ("n_free", _i(2), "n_free"), ("cu_new", _i(3), "cu_new"), ("state", _i(1), "state"),
            ("slots", _i(7).long(), "slots must be"), ("kv_lens", None, "kv_lens"),
            ("state", _i(2), "must be on a GPU")]:
        with pytest.raises(ValueError, match=re.escape(msg)):
            B.page_map(**{**ok, name: value})
    ok = dict(k=_b(5, 2, 64), v=_b(5, 2, 64), slots=_i(5), k_cache=_b(3, 2, 16, 64),
              v_cache=_b(3, 2, 16, 64))
    for name, value, msg in [
            ("k", _b(5, 2, 64).float(), "k must be a bfloat16"), ("v", _b(5, 128), "v must be ["),
            ("v", _b(4, 2, 64), "differ"), ("k", _b(5, 64, 2).transpose(1, 2), "last dimension"),
            ("slots", _i(4), "slots must be"), ("k_cache", _b(3, 2, 64), "k_cache"),
            ("v_cache", _b(4, 2, 16, 64), "v_cache"), ("slots", _i(5), "must be on a GPU")]:
        with pytest.raises(ValueError, match=re.escape(msg)):
            B.kv_cache_write(**{**ok, name: value})
    ok = dict(q=_b(3, 4, 64), k_cache=_b(3, 2, 16, 64), v_cache=_b(3, 2, 16, 64), o=_b(3, 4, 64),
              lse=torch.zeros(4, 3), kv_lens=_i(3), cu_q=None, block_table=_i(3, 2),
              prefix_pages=None, prefix_len=0, softmax_scale=0.1, softcap=None, slopes=None,
              workspace=None)
    for name, value, msg in [
            ("q", _b(3, 256), "q must be"), ("q", _b(4, 3, 64).transpose(0, 1), "contiguous"),
            ("o", _b(3, 4, 64).half(), "o must be bf16 or fp32"), ("o", _b(2, 4, 64), "o must be"),
            ("lse", torch.zeros(3, 4), "lse"), ("kv_lens", _i(2), "3 rows for 2 requests"),
            ("cu_q", _i(3), "cu_q"), ("block_table", _i(2, 2), "block_table"),
            ("prefix_len", -1, "prefix_len"), ("prefix_len", 3, "prefix_pages"),
            ("k_cache", _b(3, 2, 16, 128), "head_dim 128"),
            ("v_cache", _b(3, 2, 32, 64), "v_cache"), ("slopes", torch.zeros(3), "slopes"),
            ("lse", None, "must be on a GPU")]:
        with pytest.raises(ValueError, match=re.escape(msg)):
            B.paged_attn_fwd(**{**ok, name: value})


def test_scored_binding_checks():
    words, info = B.ta_build_schedule("causal", [0, 3], 0, 1, 0, 64)
    q, sched = _b(3, 4, 64), torch.from_numpy(words)
    with pytest.raises(ValueError, match="must be on a GPU"):
        B.scored_attn_fwd(q, _b(3, 2, 64), _b(3, 2, 64), q.clone(), None, sched, info, 0.1, 5.0,
                          None, None)
    with pytest.raises(ValueError, match="q must be bfloat16"):
        B.scored_attn_fwd(q.float(), _b(3, 2, 64), _b(3, 2, 64), q.clone(), None, sched, info, 0.1,
                          5.0, None, None)


def test_paged_positions_stay_in_32_bits():
    """Tables whose last step of keys would end past 2^31."""
    far = FAKE + (1 << 40)  # half a gigabyte and more: behind every other argument
    kw = dict(batch=1, total=1, table=far, hq=1, hkv=1)
    for width, page in (((1 << 27) - 1, 16), ((1 << 27) - 16, 16), ((1 << 23) - 1, 256)):
        assert _paged(width=width, page=page, **kw) == B.TA_ERR_UNSUPPORTED, (width, page)
        assert "32 bits" in B.ta_last_error()
    # the longest tables pass that check (and fail a later one)
    assert _paged(width=(1 << 27) - 17, q=0, **kw) == B.TA_ERR_INVALID_ARG
    assert _paged(width=(1 << 23) - 2, page=256, q=0, **kw) == B.TA_ERR_INVALID_ARG


def test_paged_distances_stay_in_32_bits():
    """With slopes, distances from the prefix's first key are counted too."""
    def call(slopes, prefix_len):
        far = FAKE + (1 << 40)
        return B.lib().paged_attn_fwd(
            None, P(FAKE), P(FAKE + M), P(FAKE + 2 * M), 0, None, P(FAKE + 3 * M), None, P(far), 1,
            1 << 22, P(far * 2), prefix_len, 1, 1, 1, 64, 9, 256, 0.1, 0.0, P(slopes),
            P(FAKE + 4 * M), 1 << 40, None)

    rest = 2 ** 31 - 257 - (1 << 30)
    assert call(FAKE + 5 * M, rest + 1) == B.TA_ERR_UNSUPPORTED
    assert call(FAKE + 5 * M, rest) == B.TA_ERR_INVALID_ARG  # q is NULL
    assert call(0, rest + 1) == B.TA_ERR_INVALID_ARG


def test_paged_launches_stay_in_32_bits():
    """More kv heads than a launch's threads hold: refused before any work."""
    kw = dict(q=0, d=64, page=16, width=1)
    assert _paged(hq=1 << 24, hkv=1 << 24, total=1, batch=1, **kw) == B.TA_ERR_UNSUPPORTED
    assert "grid" in B.ta_last_error()
    # the join of 1257 row tiles behind a prefix
    kw.update(prefix=FAKE + 7 * M, prefix_len=5, batch=1000, total=33000)
    assert _paged(hq=4096, hkv=4096, **kw) == B.TA_ERR_UNSUPPORTED
    assert "grid" in B.ta_last_error()
    assert _paged(hq=1024, hkv=1024, **kw) == B.TA_ERR_INVALID_ARG  # q is NULL
