"""The definitions of the decoder's operators in numpy, in 64 bits, and their 4-bit formats place by place.  Shares no code with the GPU path."""
import numpy as np


def groups_int4(W, group):
    """codes [N, K] int8 and scales [N, K / group] fp16 of fp32 W: IEEE fp32 arithmetic"""
    N, K = W.shape
    g = W.reshape(N, K // group, group)
    with np.errstate(all="ignore"):
        most = np.fmax.reduce(np.abs(g), axis=2, initial=np.float32(0))  # (NaN left out)
        s = np.minimum(most / np.float32(7), np.float32(65504)).astype(np.float16)
        s[s == 0] = 1
        q = g / s.astype(np.float32)[..., None]
        c = np.where(np.isnan(q), 0, np.clip(np.rint(q), -7, 7))
    return c.reshape(N, K).astype(np.int8), s


def pack_int4(codes, scales, group):
    N, K = codes.shape
    nt, kt, per = -(-N // 16), -(-K // 128), 128 // group
    out = np.zeros((nt, kt, 64, 4), np.uint32)
    for lane in range(64):
        for j in range(4):
            for e in range(8):
                n, k = np.arange(nt)[:, None] * 16 + lane % 16, np.arange(kt)[None] * 128 + 32 * j + 8 * (lane // 16) + e
                there = (n < N) & (k < K)
                c = np.where(there, codes[np.minimum(n, N - 1), np.minimum(k, K - 1)], 0).astype(np.int64) + 8
                out[:, :, lane, j] |= ((c & 15) << (e // 2 * 4 + e % 2 * 16)).astype(np.uint32)
    s = np.zeros((nt, kt * per, 16), np.float16)
    n = np.arange(nt)[:, None] * 16 + np.arange(16)[None]
    for g in range(K // group):
        s[:, g, :] = np.where(n < N, scales[np.minimum(n, N - 1), g], 0)
    return np.concatenate([out.reshape(-1).view(np.uint8), s.reshape(-1).view(np.uint8)])


def padded(D):
    return 64 if D <= 64 else 128 if D <= 128 else 256


def round7(s):
    """fp32 scale with 7 significant bits, as fp16"""
    m, e = np.frexp(s.astype(np.float64))
    with np.errstate(all="ignore"):
        s = np.where(np.isfinite(s), np.ldexp(np.rint(m * 128) / 128, e), np.inf)
    s = np.minimum(s, 896).astype(np.float16)
    return np.where(s == 0, np.float16(1), s)


def cache_codes(x):
    """x [..., D] fp32 -> codes [..., D] int and scales [..., ceil(D / 32)] fp16"""
    D = x.shape[-1]
    n = -(-D // 32)
    g = np.zeros(x.shape[:-1] + (n * 32,), np.float32)
    g[..., :D] = x
    g = g.reshape(x.shape[:-1] + (n, 32))
    with np.errstate(all="ignore"):
        s = round7(np.fmax.reduce(np.abs(g), axis=-1, initial=np.float32(0)) / np.float32(7))
        q = g / s.astype(np.float32)[..., None]
        c = np.where(np.isnan(q), 0, np.clip(np.rint(q), -7, 7))
    return c.reshape(x.shape[:-1] + (n * 32,))[..., :D].astype(np.int64), s


class Places:
    """Where a page of one head keeps a code or a scale: byte, shift, and 16-bit place"""

    def __init__(self, D):
        DP = padded(D)
        J, CH = DP // 32, DP // 16
        t, d = np.arange(64)[:, None], np.arange(DP)[None]
        self.D, self.DP, self.bytes = D, DP, 72 * DP
        self.k_byte = t * (DP // 2) + (d % 32 // 8 * J + d // 32) * 4 + d % 2 * 2 + d % 8 // 4
        self.k_shift = d % 8 // 2 % 2 * 4 + 0 * t
        self.v_byte = 36 * DP + 2 * ((((t // 4) * 16 + d // CH) * 2 + t % 4 // 2) * (DP // 64) * 2 + d % CH // 4 * 2 + t % 2) + d % 4 // 2
        self.v_shift = d % 2 * 4 + 0 * t
        g = np.arange(J)[None]
        self.k_scale = 16 * DP + t * J + g
        self.v_scale = 34 * DP + g * 64 + t


def write_pages(ck, sk, cv, sv, D, fill=0):
    """codes [pages, heads, 64, D], scales [pages, heads, 64, groups] -> pages [pages, heads, bytes] uint8"""
    p = Places(D)
    pages, heads = ck.shape[:2]
    out = np.full((pages, heads, p.bytes), fill, np.uint8)
    halves = out.view(np.uint16)
    for codes, byte, shift in ((ck, p.k_byte, p.k_shift), (cv, p.v_byte, p.v_shift)):
        full = np.zeros((pages, heads, 64, p.DP), np.int64)
        full[..., :D] = codes
        for s in (0, 4):
            sel = shift == s
            at = byte[sel]
            out[..., at] = (out[..., at] & (0xF0 if s == 0 else 0x0F)) | ((full[..., sel] + 8) << s).astype(np.uint8)
    groups = sk.shape[-1]
    for sc, at in ((sk, p.k_scale), (sv, p.v_scale)):
        full = np.ones((pages, heads, 64, p.DP // 32), np.float16)
        full[..., :groups] = sc
        halves[..., at] = full.view(np.uint16)
    return out


def read_pages(pages, D):
    """pages [.., bytes] -> K, V [.., 64, D] in 64 bits"""
    p = Places(D)
    halves = pages.view(np.float16)
    K = ((pages[..., p.k_byte] >> p.k_shift) & 15).astype(np.float64) - 8
    V = ((pages[..., p.v_byte] >> p.v_shift) & 15).astype(np.float64) - 8
    rep = lambda at: halves[..., at].astype(np.float64).repeat(32, -1)  # noqa: E731
    with np.errstate(all="ignore"):
        return (K * rep(p.k_scale))[..., :D], (V * rep(p.v_scale))[..., :D]


def norm_rope(x, norm, weight, eps, cos, sin, R, interleaved):
    """x [T, heads, D] in 64 bits; cos, sin [T, R / 2]"""
    y = x.astype(np.float64)
    if norm:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        if weight is not None:
            y = y * weight.astype(np.float64)
    if R:
        i = np.arange(R // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        c, s = cos.astype(np.float64)[:, None], sin.astype(np.float64)[:, None]
        u, v = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = u * c - v * s, u * s + v * c
    return y


def attend(q, K, V, seen, scale):
    """One head: q [n, D], K, V [S, D], seen [n, S] -> output [n, D] and how far a kernel may be off by its own roundings [n, D].

    The weights are rounded to fp16, 2^-11 of each, and below 2^-14 (the largest stands at 2^6 at least) by 2^-25; the output to fp16.  A score
    is a sum of D products in 32 bits, off by D 2^-24 of the sum of magnitudes at most, and so is its weight relative to the others, twice
    (numerator and denominator); 2^-20 covers the exponential and the other 32-bit sums, of up to 2^-24 a step over steps that are few."""
    n, D = q.shape
    out, off = np.zeros((n, D)), np.full((n, D), 2.0 ** -24)
    for i in range(n):
        k, v = K[seen[i]], V[seen[i]]
        if not len(k):
            continue
        with np.errstate(all="ignore"):
            s = (k @ q[i]) * scale
            w = np.exp(s - s.max())
            w = w / w.sum()
            out[i] = w @ v
            delta = 2 * D * 2.0 ** -24 * scale * (np.abs(k) @ np.abs(q[i]))
            off[i] += w @ (np.abs(v) * (2.0 ** -11 + 2.0 ** -20 + delta + w @ delta)[:, None]) + 2.0 ** -31 * np.abs(v).sum(0) + 2.0 ** -11 * np.abs(out[i])
    return out, off
