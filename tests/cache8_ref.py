"""Plain forms of the 8-bit cache for its tests: quantisation by search in the
list of e4m3 values, and a cache whose places that hold no key hold codes and
scales that are no numbers.

The attention's tolerances are those of the bf16 cache (tests/serving_ref.py):
held values are exact in bf16 (four significant bits, exponents of -109 and
more), a score is the same sum of products, and a value's scale, a power of two,
rounds neither the probability that it multiplies nor the product."""
import math

import numpy as np
import torch

from tests.serving_ref import Cache

E4M3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
LEAST_E, MOST_E = -100, 120


def quantise(x):
    """Rows [.., d]: (codes uint8 [.., d], scale bytes uint8 [..])."""
    x = x.detach().cpu().double().numpy()
    fine = np.isfinite(x)
    top = np.where(fine, np.abs(x), 0.0).max(-1)
    m, e = np.frexp(top / 448.0)  # top <= 448 2^e: a power of two itself is enough
    e = np.where(m > 0.5, e, e - 1)
    e = np.maximum(np.where(top > 0, e, LEAST_E), LEAST_E)
    y = np.abs(np.where(fine, x, 0.0)) * np.exp2(-e.astype(np.float64))[..., None]
    mid = (E4M3[1:] + E4M3[:-1]) / 2
    code = np.searchsorted(mid, y, side="left")  # a tie goes down here
    tie = (code < 126) & (y == mid[np.minimum(code, 125)]) & (code % 2 == 1)
    code = code + tie
    code = np.where((e == MOST_E)[..., None], np.minimum(code, np.searchsorted(E4M3, 240.0)), code)
    code = np.where(np.signbit(x), code + 128, code)
    code = np.where(fine, code, 127)
    return (torch.from_numpy(code.astype(np.uint8)),
            torch.from_numpy((e + 127).astype(np.uint8)))


def values(codes, scales):
    """What codes [.., d] and scale bytes [..] stand for, in 64 bits."""
    two = torch.exp2(scales.double() - 127.0)
    two = torch.where(scales == 255, math.nan, two)
    return codes.view(torch.float8_e4m3fn).double() * two[..., None]


def typed(codes, scales):
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)


class Cache8(Cache):
    """A Cache held in 8 bits: k and v are the held values in bf16, k8, ks, v8
    and vs the codes and scale bytes."""

    def __init__(self, lens, hkv, d, page, prefix=0, seed=0, spare=3, device="cuda", sink=8.0):
        super().__init__(lens, hkv, d, page, prefix, seed, spare, "cpu", sink)
        g = torch.Generator().manual_seed(seed + 1)
        size = torch.exp2(torch.randint(-6, 3, (hkv, 1, 1), generator=g).float())
        for name in ("k", "v"):
            x = getattr(self, name)
            if name == "v":
                x = x * size.bfloat16()  # heads of different sizes
            codes, scales = quantise(x)
            none = torch.isnan(x).all(-1)  # a place that holds no key
            codes[none], scales[none] = 255, 255
            setattr(self, name, values(codes, scales).bfloat16().to(device))
            setattr(self, name + "8", codes.to(device))
            setattr(self, name + "s", scales.to(device))
        self.table, self.kv_lens = self.table.to(device), self.kv_lens.to(device)
        self.prefix_pages = self.prefix_pages.to(device)

    def tensors(self):
        """(k_cache, v_cache, {k_scale, v_scale}) of a call."""
        k, ks = typed(self.k8, self.ks)
        v, vs = typed(self.v8, self.vs)
        return k, v, dict(k_scale=ks, v_scale=vs)

    def put(self, name, page, place, head=0, code=None, at=None, scale=None):
        """Another code or scale byte of one row, held values too."""
        if code is not None:
            getattr(self, name + "8")[page, head, place, at] = code
        if scale is not None:
            getattr(self, name + "s")[page, head, place] = scale
        getattr(self, name)[page, head, place] = values(
            getattr(self, name + "8")[page, head, place],
            getattr(self, name + "s")[page, head, place]).bfloat16()
