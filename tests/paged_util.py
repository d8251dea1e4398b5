"""Plain forms in 64 bits of attention, of the 8-bit pages and of their bookkeeping, and how far a kernel may be from them."""
import numpy as np
import torch

PAGE = 64
#: half a step of a rounding to the type, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def attend(q, k, v, seen, scale, dtype):
    """q [R, hd], k / v [S, hd] (64 bits), seen [R, S] bool: (result [R, hd], bound of a kernel's distance from it).

    The bound adds up what a kernel with 32-bit sums does: a score is a sum of hd products (hd + 8 roundings of 2^-24 of the sum of their
    magnitudes, scale and exponential included; the exponential's own error is under 2^-20), P is rounded once to the type, sums over
    S slots add S + 64 roundings of 2^-24 (the joins of waves and splits among them) in the numerator and in the denominator, and the
    result is rounded once to the type.  A = sum p |v| / sum p carries all but the last."""
    hd, S = q.shape[1], k.shape[0]
    use = seen.any(dim=0)
    s = torch.where(seen, (q @ torch.where(use[:, None], k, 0.0).T.contiguous()) * scale, -torch.inf)
    top = s.amax(dim=1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0.0))
    vz = torch.where(use[:, None], v, 0.0)
    # a slot that some row sees counts for the rows that see it alone
    odd = ~torch.isfinite(vz).all(dim=1)
    num, den = p @ torch.where(odd[:, None], 0.0, vz), p.sum(dim=1, keepdim=True)
    for j in torch.nonzero(odd)[:, 0].tolist():
        num = torch.where(seen[:, j, None], num + p[:, j, None] * vz[j], num)
    none = ~seen.any(dim=1, keepdim=True)
    o = torch.where(none, 0.0, num / den)
    A = torch.where(none, 0.0, (p @ torch.where(torch.isfinite(vz), vz, 0.0).abs()) / den)
    mag = (q.abs() @ torch.where(torch.isfinite(k) & use[:, None], k, 0.0).abs().T.contiguous()).amax(dim=1, keepdim=True) * scale
    delta = 2 * (hd + 8) * 2.0 ** -24 * torch.where(torch.isfinite(mag), mag, 0.0) + 2 * 2.0 ** -20 + 2 * (S + 64) * 2.0 ** -24
    once = HALF[dtype] if dtype != torch.float32 else 0.0
    return o, A * (once + delta) * 1.02 + o.abs() * HALF[dtype] * 1.01 + 1e-37


def check(got, want, tol, what):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()), float((got - want).abs()[fine].max()))


def nearest_e4m3(y):
    """64-bit numpy values to the nearest e4m3 value (ties to even), magnitudes up to 448."""
    a = np.abs(y)
    _, e = np.frexp(a)  # a = m 2^e, m in [1/2, 1)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.sign(y) * np.rint(a / step) * step


def exponent(top):
    """The smallest e >= -117 with top <= 448 * 2^e, by trying them."""
    e = -117
    while top > np.ldexp(448.0, e):
        e += 1
    return e


def quantise(rows):
    """rows [n <= 64, hd] of one tile, 64 bits: (values over the scale [64, hd], scale)."""
    full = np.zeros((PAGE, rows.shape[1]))
    full[:rows.shape[0]] = rows
    fine = np.isfinite(full)
    e = exponent(np.abs(np.where(fine, full, 0.0)).max())
    return np.where(fine, nearest_e4m3(np.ldexp(np.where(fine, full, 0.0), -e)), np.nan), np.ldexp(1.0, e)


def values(pool_codes, pool_scales, page, layer, hd):
    """(K, V) [heads, 64, hd] in 64 bits that a page stands for, read by the documented places one by one."""
    c = pool_codes[page, layer].view(torch.float8_e4m3fn).double().cpu().numpy()  # [2, heads, 64 * hd]
    s = pool_scales[page, layer].double().cpu().numpy()
    heads = c.shape[1]
    k, v = np.empty((heads, PAGE, hd)), np.empty((heads, PAGE, hd))
    for t in range(PAGE):
        for a in range(hd // 64):
            k[:, t, 64 * a:64 * a + 64] = c[0, :, (a * PAGE + t) * 64:(a * PAGE + t) * 64 + 64]
        v[:, t] = c[1, :, np.arange(hd) * PAGE + 16 * ((t >> 2) & 3) + 4 * (t >> 4) + (t & 3)].T
    return k * s[0][:, None, None], v * s[1][:, None, None]


class HostPool:
    """The bookkeeping on the host, one step after another."""

    def __init__(self, n_pages, n_seqs, max_pages):
        self.ref, self.length = np.zeros(n_pages, np.int32), np.zeros(n_seqs, np.int32)
        self.table = np.full((n_seqs, max_pages), -1, np.int32)

    def _free(self):
        return np.nonzero(self.ref == 0)[0]

    def grow(self, seqs, n_tokens):
        if any(n < self.length[s] for s, n in zip(seqs, n_tokens)):
            return -2
        need = [-(-n // PAGE) - -(-int(self.length[s]) // PAGE) for s, n in zip(seqs, n_tokens)]
        if sum(need) > len(self._free()):
            return -1
        for s, n, m in zip(seqs, n_tokens, need):
            have = -(-int(self.length[s]) // PAGE)
            for i in range(m):
                p = self._free()[0]
                self.table[s, have + i], self.ref[p] = p, 1
            self.length[s] = n
        return sum(need)

    def fork(self, src, dst):
        """Returns the status and the (old, new) pages whose contents are copied."""
        if any(self.length[d] for d in dst):
            return -2, []
        if sum(int(self.length[s]) % PAGE > 0 for s in src) > len(self._free()):
            return -1, []
        moves = []
        for s, d in zip(src, dst):
            n = int(self.length[s])
            self.table[d] = -1
            for i in range(-(-n // PAGE)):
                p = self.table[s, i]
                if (i + 1) * PAGE > n:
                    new = self._free()[0]
                    moves.append((int(p), int(new)))
                    p = new
                self.ref[p] += 1
                self.table[d, i] = p
            self.length[d] = n
        return len(moves), moves

    def free(self, seqs):
        for s in seqs:
            for p in self.table[s][self.table[s] >= 0]:
                self.ref[p] -= 1
            self.table[s], self.length[s] = -1, 0

    def compact(self):
        live, moves = int((self.ref > 0).sum()), []
        for p in range(live, len(self.ref)):
            if self.ref[p] > 0:
                new = int(self._free()[0])
                self.ref[new], self.ref[p] = self.ref[p], 0
                self.table[self.table == p] = new
                moves.append((p, new))
        return moves
