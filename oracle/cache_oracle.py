"""CPU oracle for the paged cache's bookkeeping and for its 8-bit pages.  TEST INFRASTRUCTURE ONLY.

Plain Python / numpy, one entry at a time, written from the definitions in include/lorc.h; it shares no code with the library.
"""
from __future__ import annotations

import numpy as np

PAGE, GROUP = 64, 128
OK, REFUSED, SHORT = 0, 1, 2


# =============================================================================== pages
class Pages:
    """A block table and the counts of its pages.  All calls are the definitions, in order of the lists."""

    def __init__(self, table, refs):
        self.table, self.refs = np.array(table, np.int32), np.array(refs, np.int32)

    def maps(self, i):
        return 0 <= i < len(self.refs)

    def _free(self):
        return [int(i) for i in np.flatnonzero(self.refs <= 0)]

    def fork(self, parents, children, lens):
        n_seqs, max_pages = self.table.shape
        valid = [0 <= p < n_seqs and 0 <= c < n_seqs and p != c and 0 <= L <= PAGE * max_pages
                 for p, c, L in zip(parents, children, lens)]
        named = {c for v, c in zip(valid, children) if v}
        before, free, seen = self.table.copy(), self._free(), set()
        src, dst, status = [], [], []
        for v, p, c, L in zip(valid, parents, children, lens):
            src.append(-1), dst.append(-1)
            if not v or c in seen or p in named or self.maps(before[c, 0]):
                status.append(REFUSED)
                if v:
                    seen.add(c)
                continue
            seen.add(c)
            tail = int(before[p, L // PAGE]) if L % PAGE else -1
            if self.maps(tail):
                if not free:
                    status.append(SHORT)
                    continue
                src[-1], dst[-1] = tail, free.pop(0)
            status.append(OK)
            for e in range(len(self.table[c])):
                if self.maps(before[c, e]):
                    self.refs[before[c, e]] -= 1
            self.table[c] = -1
            for e in range(L // PAGE):
                if self.maps(before[p, e]):
                    self.table[c, e] = before[p, e]
                    self.refs[before[p, e]] += 1
            if dst[-1] >= 0:
                self.table[c, L // PAGE] = dst[-1]
                self.refs[dst[-1]] = 1
        return src, dst, status

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.table):
                for e in range(self.table.shape[1]):
                    if self.maps(self.table[s, e]):
                        self.refs[self.table[s, e]] -= 1
                    self.table[s, e] = -1

    def compact(self, max_moves):
        src, dst, new = [], [], np.arange(len(self.refs), dtype=np.int32)
        free, used = self._free(), [int(i) for i in np.flatnonzero(self.refs > 0)][::-1]
        for hole, page in zip(free, used):
            if hole > page or len(src) == max_moves:
                break
            src.append(page), dst.append(hole)
            new[page] = hole
            self.refs[hole], self.refs[page] = self.refs[page], 0
        for i, v in np.ndenumerate(self.table):
            if self.maps(v):
                self.table[i] = new[v]
        fill = [-1] * (max_moves - len(src))
        return src + fill, dst + fill, new

    def reserve(self, seqs, lens):
        n_seqs, max_pages = self.table.shape
        free, seen, status, short = self._free(), set(), [], False
        for s, L in zip(seqs, lens):
            if not (0 <= s < n_seqs and 0 <= L <= PAGE * max_pages) or s in seen:
                status.append(REFUSED)
                continue
            seen.add(s)
            missing = [e for e in range(-(-L // PAGE)) if not self.maps(self.table[s, e])]
            if missing and (short or len(missing) > len(free)):
                short = True
                status.append(SHORT)
                continue
            for e in missing:
                self.table[s, e] = free.pop(0)
                self.refs[self.table[s, e]] = 1
            status.append(OK)
        return status


# =============================================================================== 8-bit pages
def e4m3_values():
    """The 256 codes of OCP e4m3: sign, four bits of exponent (bias 7), three of fraction; S.1111.111 is NaN, there is no infinity."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


def encode(x):
    """Round to the nearest e4m3 value, ties to the even code; NaN and infinities -> NaN.  |x| <= 448 (larger finite values are not defined)."""
    x = np.asarray(x, np.float64)
    mags = e4m3_values()[:127]
    a = np.abs(x)
    fine = np.isfinite(x)
    i = np.clip(np.searchsorted(mags, np.where(fine, a, 0.0)), 0, 126)
    low = np.maximum(i - 1, 0)
    d_hi, d_lo = mags[i] - a, a - mags[low]
    take_low = (d_lo < d_hi) | ((d_lo == d_hi) & (low % 2 == 0))
    code = np.where(take_low & (i > 0), low, i)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(fine, code, np.where(np.signbit(x), 255, 127)).astype(np.uint8)


def scale_exponents(x):
    """Least k >= -126 with (largest finite magnitude of the group) <= 448 * 2^k, for every group of 128 of the last axis."""
    r = x.shape[-1]
    out = []
    for g in range(0, r, GROUP):
        a = np.abs(np.asarray(x[..., g:g + GROUP], np.float64))
        a = np.where(np.isfinite(a), a, 0.0).max(-1)
        k = np.full(a.shape, -126)
        while np.any(a > 448.0 * 2.0 ** k):
            k = np.where(a > 448.0 * 2.0 ** k, k + 1, k)
        out.append(k)
    return np.stack(out, -1)


def quantize(x):
    """[..., r] -> (codes uint8 [..., r], exponents [..., groups])."""
    x = np.asarray(x, np.float64)
    k = scale_exponents(x)
    return encode(x / 2.0 ** np.repeat(k, GROUP, -1)[..., :x.shape[-1]].astype(np.float64)), k


def dequantize(codes, k):
    return e4m3_values()[codes] * 2.0 ** np.repeat(k, GROUP, -1)[..., :codes.shape[-1]].astype(np.float64)


def page_size(r_k, r_v):
    groups = -(-r_k // GROUP) + -(-r_v // GROUP)
    return PAGE * (r_k + r_v + groups)


def scale_index(r_k, r_v, slot, j, value):
    """Byte of an 8-bit page that scales K latent j of a slot, or (value) V latent j."""
    first = -(-r_k // GROUP) if value else 0
    return PAGE * (r_k + r_v) + (first + j // GROUP) * PAGE + slot
