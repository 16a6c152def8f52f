"""The definitions of the operators that answer with drafted tokens, in numpy, in 64 bits.  Shares no code with the GPU path."""
import numpy as np

import decoder_reference as ref


def chain(parents, i):
    """Node i and all that it follows; what is no node in front of it is no parent"""
    out = [i]
    while 0 <= parents[out[-1]] < out[-1]:
        out.append(int(parents[out[-1]]))
    return out


def bits(rows, words):
    """Lists of nodes -> [rows, words] int32"""
    out = np.zeros((len(rows), words), np.uint32)
    for i, nodes in enumerate(rows):
        for j in nodes:
            out[i, j // 32] |= np.uint32(1 << (j % 32))
    return out.view(np.int32)


def slots(table, place):
    """A table's row: where its tokens are"""
    ok = 0 <= place < 64 * len(table) and 0 <= table[place // 64] < 2**25
    return int(table[place // 64]) * 64 + place % 64 if ok else -1


def accepted(parents, drafted, sampled):
    """Nodes that are kept, the token behind the last"""
    if not len(parents):
        return [], -1
    kept = [0]
    while sampled[kept[-1]] >= 0:
        more = [i for i in range(kept[-1] + 1, len(parents)) if parents[i] == kept[-1] and drafted[i] == sampled[kept[-1]]]
        if not more:
            break
        kept.append(more[0])
    return kept, int(sampled[kept[-1]])


def moved(pages, D, pairs):
    """pages [num, heads, bytes]: tokens (from, to), in slots, read before any is written"""
    p = ref.Places(D)
    out, halves = pages.copy(), pages.view(np.uint16)
    to_halves = out.view(np.uint16)
    for a, b in pairs:
        if a < 0 or b < 0:
            continue
        (pa, ta), (pb, tb) = divmod(a, 64), divmod(b, 64)
        for byte in (p.k_byte, p.v_byte):  # (both codes of a byte are of one token)
            out[pb][:, byte[tb]] = pages[pa][:, byte[ta]]
        for at in (p.k_scale, p.v_scale):
            to_halves[pb][:, at[tb]] = halves[pa][:, at[ta]]
    return out


def tokens8(X, Wq, w_scale, bias, gelu):
    """X fp16 or fp32 -> output in 64 bits, and how far 32-bit arithmetic behind the exact sum may be off (in front of the output's rounding):
    the sum as fp32, its product with the token's scale, and the fused step with the channel's: 2^-24 each of what they have; GELU's slope is at most
    1.13, its own error a few 2^-24"""
    X = X.astype(np.float32)
    most = np.fmax.reduce(np.abs(X), axis=1, initial=np.float32(0))
    s = np.where(most == 0, np.float32(1), most / np.float32(127)).astype(np.float32)[:, None]
    with np.errstate(all="ignore"):
        q = X / s
        q = np.where(np.isnan(q), 0, np.clip(np.rint(q), -127, 127)).astype(np.float64)
    y = (q @ Wq.T.astype(np.float64)) * s.astype(np.float64) * w_scale.astype(np.float64)
    off = 2 * 2.0 ** -24 * np.abs(y)
    if bias is not None:
        y = y + bias.astype(np.float64)
    off = off + 2.0 ** -24 * np.abs(y) + 2.0 ** -148
    if gelu:
        from scipy.special import ndtr
        y = y * ndtr(y)
        off = 1.13 * off + 2.0 ** -20 * np.abs(y) + 1e-30
    return y, off * (1 + 2.0 ** -20)


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row, parameters as the fp32 (int32) numbers they are -> token, its share, and how close u comes to another token's share, relative to all"""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    top = x.max()
    if top == -np.inf:
        return -1, 0.0, np.inf
    if not temperature > 0:
        return int(np.argmax(x)), 1.0, np.inf
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / np.float64(temperature)))
    w[~(w >= 2.0 ** -40)] = 0.0
    order = np.lexsort((np.arange(len(x)), -x))
    n = top_k if 0 < top_k < len(x) else len(x)
    if top_p < 1:
        mass = np.cumsum(w[order[:n]])
        n = max(1, int(np.searchsorted(mass, np.float64(top_p) * mass[-1], side="left")) + 1)
    keep = np.zeros(len(x), bool)
    keep[order[:n]] = True
    keep &= (w > 0) & (w >= min(np.float64(min_p), 1.0))
    w[~keep] = 0.0
    upto = np.cumsum(w)
    token = int(np.searchsorted(upto, np.float64(u) * upto[-1], side="right"))
    if token == len(x):
        token = int(np.nonzero(keep)[0][-1])
    return token, w[token] / upto[-1], np.abs(upto[keep] / upto[-1] - u).min()
