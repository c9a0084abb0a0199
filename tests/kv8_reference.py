"""The 8-bit key/value cache and the token log probabilities written out in 64 bits on the CPU."""
import numpy as np

E_MIN, E_MAX, LARGEST = -63, 63, 448.0 * 2.0 ** 63


def e4m3_table():
    """The 256 numbers of the e4m3 format."""
    out = np.zeros(256)
    for c in range(256):
        s, e, f = (-1.0 if c & 128 else 1.0), (c >> 3) & 15, c & 7
        out[c] = s * (f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10))
        if c & 127 == 127:
            out[c] = np.nan
    return out


TABLE = e4m3_table()


def encode(y):
    """e4m3 codes of y (|y| <= 448 or NaN), to nearest, ties to the even fraction, by search in the table."""
    y = np.asarray(y, np.float64)
    pos = TABLE[:127]
    a = np.abs(np.where(np.isnan(y), 0.0, y))
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.clip(hi - 1, 0, 126)
    dl, dh = a - pos[lo], pos[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.signbit(y), pick + 128, pick)
    return np.where(np.isnan(y), 127, code).astype(np.uint8)


def needed_exponent(a):
    e = E_MIN
    while a > 448.0 * 2.0 ** e:
        e += 1
    return e


class Cache:
    """codes uint8 [2, pages, heads, page_tokens, head_dim], exponents int [pages, heads, 2]."""

    def __init__(self, codes, scales):
        self.codes = np.array(codes)
        with np.errstate(divide="ignore"):
            self.e = np.clip(np.nan_to_num(np.log2(np.array(scales, np.float64)), neginf=-1000), E_MIN, E_MAX).round().astype(int)
        self.touched = np.zeros(self.e.shape, bool)
        self.page = self.codes.shape[3]

    def write(self, pages, pos0, x, which):
        """x [n, heads, head_dim] at positions pos0 .. of the sequence whose pages these are."""
        n = len(x)
        for j in range(pos0 // self.page, -(-(pos0 + n) // self.page)):
            lo, hi = max(pos0, j * self.page), min(pos0 + n, (j + 1) * self.page)
            pg, slot = pages[j], lo - j * self.page
            for h in range(x.shape[1]):
                new = np.asarray(x[lo - pos0:hi - pos0, h], np.float64)
                fine = np.abs(np.where(np.isfinite(new), new, np.inf)) <= LARGEST
                e = needed_exponent(np.abs(new[fine]).max() if fine.any() else 0.0)
                if slot:
                    old = self.e[pg, h, which]
                    e = max(e, old)
                    self.codes[which, pg, h, :slot] = encode(TABLE[self.codes[which, pg, h, :slot]] * 2.0 ** (old - e))
                self.codes[which, pg, h, slot:slot + hi - lo] = encode(np.where(fine, np.where(fine, new, 0.0) * 2.0 ** -e, np.nan))
                self.e[pg, h, which] = e
                self.touched[pg, h, which] = True

    def values(self, pages, n, which):
        """[n, heads, head_dim]"""
        pages = list(pages[: -(-n // self.page)])
        x = TABLE[self.codes[which, pages]] * 2.0 ** self.e[pages, :, which][:, :, None, None]
        return x.transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:n]


def attention(q, k, v, first, scale, size=None):
    """q [n, heads, d] at positions first ..; k, v [length, kv_heads, d].  Returns o, and for error bounds
    sum_j p_j |v_j|, and per (row, head) the largest scale * sum_d |q_d k_jd| and (with size [length, kv_heads], the
    scales that the values were stored with) the largest p_j * size_j."""
    n, H, d = q.shape
    g = H // k.shape[1]
    o, wide, big, top = np.zeros((n, H, d)), np.zeros((n, H, d)), np.zeros((n, H)), np.zeros((n, H))
    for i in range(n):
        m = first + i + 1
        if m <= 0:
            continue
        for h in range(H):
            kk, vv, qq = k[:m, h // g], v[:m, h // g], q[i, h].astype(np.float64)
            with np.errstate(invalid="ignore", over="ignore"):
                s = kk @ qq * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                o[i, h], wide[i, h] = p @ vv, p @ np.abs(vv)
                big[i, h] = (np.abs(kk) @ np.abs(qq)).max() * abs(scale)
                if size is not None:
                    top[i, h] = (p * size[:m, h // g]).max()
    return o, wide, big, top


def logprobs(x, scale):
    """log softmax of scale * x (rows with nothing but -inf: -inf), lse and entropy.  scale * x beyond fp32 is infinite."""
    y = np.asarray(x, np.float64) * scale
    with np.errstate(over="ignore"):
        y = np.where(np.isinf(y.astype(np.float32)), y.astype(np.float32).astype(np.float64), y)
    m = y.max(1, keepdims=True)
    m0 = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(y - m0)
        lse = m0[:, 0] + np.log(e.sum(1))
        empty = np.isneginf(lse)
        lp = np.where(empty[:, None], -np.inf, y - np.where(empty, 0.0, lse)[:, None])
        p = np.exp(lp)
        ent = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(1)
    return lp, lse, np.where(np.isnan(lse), np.nan, ent)


def logprobs_grad(x, scale, targets, d_logp, d_entropy):
    lp, lse, ent = logprobs(x, scale)
    p = np.exp(lp)
    V = p.shape[1]
    g = np.zeros_like(p)
    for r in range(len(p)):
        if np.isneginf(lse[r]):
            continue
        for t, d in zip(targets[r], d_logp[r]):
            if 0 <= t < V:
                g[r] -= d * p[r]
                g[r, t] += d
        if d_entropy is not None:
            g[r] -= np.where(p[r] > 0, d_entropy[r] * p[r] * (np.where(p[r] > 0, lp[r], 0.0) + ent[r]), 0.0)
    return g * scale
