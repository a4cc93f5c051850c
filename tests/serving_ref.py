"""Plain 64-bit forms and shared helpers of the serving operators' tests.

Tolerances.  A kernel rounds each probability to bf16 for the PV product (half
a step, 2^-8 relative), which moves an output element by at most 2^-8 times
the probability-weighted mean of |v| (absw).  An error e of a score moves the
probabilities by at most 2 e relative, so that e <= 2^-13 is covered by
another 2^-12 absw; the scores here (products of 64 or 128 terms in fp32, of
size up to 60, with caps up to 50 and biases up to a few hundred at keys that
matter) stay within: 60 * 2^-24 * 16 for the sums of products in blocks of 16,
2^-22 * 50 for a cap, 2^-23 * 300 for a bias are 5.7e-5, 1.2e-5 and 3.6e-5,
together 1.05e-4 < 2^-13.  A bf16 output adds half a step of itself, 2^-8.
The log-sum-exp moves by at most e, plus the fp32 rounding of its own size.
"""
import math

import numpy as np
import torch

U = 2.0 ** -8


def o_tolerance(o, absw, dtype):
    tol = (U + 2.0 ** -12) * absw + 1e-5
    return tol + U * o.abs() if dtype == torch.bfloat16 else tol


def lse_tolerance(lse):
    return 2.0 ** -13 + 2.0 ** -22 * lse.abs()


def attend(q, k, v, keep, dist, scale, softcap=None, slopes=None):
    """q [R, hq, d] over k, v [n, hkv, d]: (o [R, hq, d], lse [R, hq], absw)
    in 64 bits.  keep, dist (row - key) [R, n].  Values of keys that a row
    does not keep are not used."""
    R, hq, d = q.shape
    group = hq // k.shape[1]
    o = torch.zeros(R, hq, d, dtype=torch.float64, device=q.device)
    absw, lse = torch.zeros_like(o), torch.full((R, hq), -math.inf, dtype=torch.float64,
                                                device=q.device)
    if k.shape[0] == 0:
        return o, lse, absw
    seen = keep.any(0)  # keys that no row keeps may hold anything
    for h in range(hq):
        kk = torch.where(seen[:, None], k[:, h // group].double(), 0.0)
        vv = torch.where(seen[:, None], v[:, h // group].double(), 0.0)
        x = q[:, h].double() @ kk.t().contiguous() * scale
        if softcap:
            x = softcap * torch.tanh(x / softcap)
        if slopes is not None:
            x = x - float(slopes[h]) * dist.double()
        x = x.masked_fill(~keep, -math.inf)
        lse[:, h] = torch.logsumexp(x, -1)
        some = keep.any(1)
        p = torch.where(some[:, None], torch.exp(x - lse[:, h:h + 1]), 0.0)
        p = p.masked_fill(~keep, 0.0)
        if torch.isfinite(vv).all():
            o[:, h], absw[:, h] = p @ vv, p @ vv.abs()
        else:
            part = torch.where(keep[:, :, None], p[:, :, None] * vv[None], 0.0)
            o[:, h], absw[:, h] = part.sum(1), part.abs().sum(1)
    return o, lse, absw


def check(o, lse, ref, dtype, label, underflow=False):
    """o [R, hq, d], lse [R, hq] or None against attend()'s result.  With
    `underflow`, an infinite value whose key has a score of 104 or more below
    the row's largest may also give NaN: e^-104 = 2^-150 is 0 in fp32, and 0
    times infinity NaN, where 64 bits hold the probability."""
    ro, rl, absw = ref
    o = o.double()
    fine = torch.isfinite(ro)
    if underflow:
        assert torch.equal(torch.isfinite(o), fine), label
    else:
        assert torch.equal(torch.isnan(o), torch.isnan(ro)), label
        assert torch.equal(o[~fine & ~torch.isnan(ro)], ro[~fine & ~torch.isnan(ro)]), label
    err = (o - ro).abs()[fine]
    tol = o_tolerance(ro, absw, dtype)[fine]
    worst = float((err / tol).max()) if err.numel() else 0.0
    assert worst <= 1.0, f"{label}: {worst:.2f} of the tolerance"
    worst_l = 0.0
    if lse is not None:
        lse = lse.double()
        assert torch.equal(torch.isfinite(lse), torch.isfinite(rl)), label
        f = torch.isfinite(rl)
        assert torch.equal(lse[~f & ~torch.isnan(rl)], rl[~f & ~torch.isnan(rl)]), label
        e = ((lse - rl).abs() / lse_tolerance(rl))[f]
        worst_l = float(e.max()) if e.numel() else 0.0
        assert worst_l <= 1.0, f"{label}: lse {worst_l:.2f} of the tolerance"
    print(f"{label}: {worst:.2f} of the tolerance, lse {worst_l:.2f}", flush=True)


class Cache:
    """A paged cache of requests with `lens` own keys behind an optional
    shared prefix; places that hold no key are NaN, table entries that name no
    page are -1."""

    def __init__(self, lens, hkv, d, page, prefix=0, seed=0, spare=3, device="cuda", sink=8.0):
        g = torch.Generator().manual_seed(seed)
        n_pre = -(-prefix // page)
        need = [-(-n // page) for n in lens]
        total = sum(need) + n_pre + spare
        order = torch.randperm(total, generator=g)
        width = max(need + [0]) + 1
        self.lens, self.page, self.prefix = lens, page, prefix
        self.table = torch.full((len(lens), width), -1, dtype=torch.int32)
        self.prefix_pages = order[:n_pre].to(torch.int32)
        kc = torch.full((total, hkv, page, d), math.nan, dtype=torch.bfloat16)
        vc = kc.clone()
        at = n_pre
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n].to(torch.int32)
            at += n

        def fill(pages, n):
            for i, p in enumerate(pages.tolist()):
                m = min(page, n - i * page)
                kc[p, :, :m] = torch.randn(hkv, m, d, generator=g).bfloat16()
                vc[p, :, :m] = torch.randn(hkv, m, d, generator=g).bfloat16()
                if i == 0:
                    kc[p, :, 0] *= sink
        fill(self.prefix_pages, prefix)
        for b, n in enumerate(lens):
            fill(self.table[b, :need[b]], n)
        self.k, self.v = kc.to(device), vc.to(device)
        self.table, self.prefix_pages = self.table.to(device), self.prefix_pages.to(device)
        self.kv_lens = torch.tensor(lens, dtype=torch.int32, device=device)

    def keys(self, b):
        """(k, v) [prefix + n, hkv, d] of request b."""
        n, page = self.lens[b], self.page
        out = []
        for c in (self.k, self.v):
            parts = []
            for pages, m in ((self.prefix_pages, self.prefix), (self.table[b], n)):
                x = c[pages[:-(-m // page)].long()].transpose(1, 2)
                parts.append(x.reshape(-1, c.shape[1], c.shape[3])[:m])
            out.append(torch.cat(parts))
        return out

    def reference(self, q, q_lens, scale, softcap=None, slopes=None):
        """attend() of every request's rows, packed: (o, lse [R, hq], absw)."""
        parts, at = [], 0
        for b, m in enumerate(q_lens):
            k, v = self.keys(b)
            n = self.lens[b]
            pos = n - m + torch.arange(m, device=q.device)
            key = torch.arange(-self.prefix, n, device=q.device)
            dist = pos[:, None] - key
            keep = (dist >= 0) & (pos >= 0)[:, None]
            parts.append(attend(q[at:at + m], k, v, keep, dist, scale, softcap, slopes))
            at += m
        return tuple(torch.cat(x) for x in zip(*parts))


def geometric_slopes(hq, device="cuda"):
    h = torch.arange(1, hq + 1, dtype=torch.float32, device=device)
    return torch.exp2(-8.0 * h / hq)


def page_map_ref(cached, new, table, free, n_free, page, slot_count):
    """ta_page_map of host lists: (table, kv_lens, cu_new, slots, state)."""
    table = [list(row) for row in table]
    width = len(table[0]) if table else 0
    up = lambda n: -(-n // page)  # noqa: E731
    bad = 0
    if n_free < 0 or n_free > len(free):
        bad |= 16
    if any(c < 0 or n < 0 for c, n in zip(cached, new)):
        bad |= 4
    cz = [c if c >= 0 and n >= 0 else 0 for c, n in zip(cached, new)]
    nz = [n if c >= 0 and n >= 0 else 0 for c, n in zip(cached, new)]
    if any(up(c + n) > width for c, n in zip(cz, nz)):
        bad |= 2
    if sum(up(c + n) - up(c) for c, n in zip(cz, nz)) > n_free:
        bad |= 1
    if sum(nz) > slot_count:
        bad |= 8
    if bad:
        return table, list(cached), [0] * (len(cached) + 1), [-1] * slot_count, [n_free, bad]
    slots, cu, taken = [], [0], 0
    for b, (c, n) in enumerate(zip(cached, new)):
        for x in range(up(c), up(c + n)):
            table[b][x] = free[n_free - 1 - taken]
            taken += 1
        for p in range(c, c + n):
            e = table[b][p // page]
            s = e * page + p % page
            slots.append(s if e >= 0 and s < 2 ** 31 else -1)
        cu.append(cu[-1] + n)
    slots += [-1] * (slot_count - len(slots))
    return (table, [c + n for c, n in zip(cached, new)], cu, slots, [n_free - taken, 0])


def scored_keep(kind, n, sink, window, last, tile=None, lists=None):
    """Kept pairs [n, n] of one sequence (numpy bool)."""
    i = np.arange(n)[:, None]
    j = np.arange(n)[None, :]
    keep = j <= i
    if kind == "triangle":
        keep &= (j < sink) | (i - j < window) | (i >= n - min(last, n))
    if kind == "blocksparse":
        on = np.zeros((-(-n // tile), -(-n // tile)), dtype=bool)
        for t, tiles in enumerate(lists):
            on[t, tiles] = True
        keep &= on[i // tile, j // tile]
    return keep
