"""Timed cases of the operators of a decoder that answers with drafted tokens, one pass of one operator each.

A small model drafts a tree of tokens behind each sequence; the decoder runs all of them in one step and keeps the branch that it would have
answered with.  Kinds of case
  draft   which drafted tokens each one follows, their positions and slots of the cache, from the tree's parents (`gpusq.draft_tree`)
  tree    attention of a tree's tokens over the paged 4-bit cache (`gpusq.attention_kv4` with `tree`)
  int8    a linear layer in 8-bit integers with scales for each token and channel: the vocabulary's, a prompt's (`gpusq.linear_int8_tokens`)
  sample  tokens drawn from logits by temperature, top-k, top-p and min-p with given random numbers (`gpusq.sample_tokens`)
  accept  the branch whose drafts are what was drawn, moved together in the layers' caches (`gpusq.accept_drafts`)

The plain forms compute in 32 bits, the masses of `sample` in 64 (a token's border is closer to the next one's than 32 bits tell apart), and round
once at the end.  exact() is the definition in 64 bits; it finds codes and scales by their places in the formats of include/gpusq.h one by
one, where the plain forms unpack whole words.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f16": torch.float16, "f32": torch.float32}
_PAGE = 64  # tokens of a page of the cache
_LEAST = 2.0**-40  # tokens of a smaller weight, of the largest one's, are not drawn


def _draft(name, B, nodes, longest):
    return dict(name=name, kind="draft", B=B, nodes=nodes, longest=longest)


def _tree(name, B, heads, kv_heads, D, longest, nodes):
    return dict(name=name, kind="tree", B=B, heads=heads, kv_heads=kv_heads, D=D, longest=longest, nodes=nodes)


def _int8(name, M, K, N, bias=True, gelu=False, x="f16", out="f16"):
    return dict(name=name, kind="int8", M=M, K=K, N=N, bias=bias, gelu=gelu, x=x, out=out)


def _sample(name, rows, V, x="f32", filters="none"):
    return dict(name=name, kind="sample", rows=rows, V=V, x=x, filters=filters)


def _accept(name, B, nodes, layers, kv_heads, D, longest):
    return dict(name=name, kind="accept", B=B, nodes=nodes, layers=layers, kv_heads=kv_heads, D=D, longest=longest)


def listed():
    return [
        # one sequence with a handful of drafts: a launch
        _draft("draft, one tree of 8", 1, 8, 2000),
        # a serving batch with wide trees
        _draft("draft, 64 trees of 61", 64, 61, 5000),
        # a small decoder's tree behind a short history: latency
        _tree("tree of 7, short history", 1, 16, 16, 64, 500, 7),
        # a serving batch: ragged histories, grouped heads
        _tree("16 trees of 24, ragged", 16, 32, 8, 128, 4096, 24),
        # one sequence with a long history and a wide tree: the work has to be split over the history
        _tree("tree of 63, long history", 1, 32, 8, 128, 65537, 63),
        # the vocabulary's logits for a tree of 9 tokens: the weights' bytes
        _int8("vocabulary, 9 tokens", 9, 4096, 131072, bias=False, out="f32"),
        # a prompt through a feed-forward layer with GELU: arithmetic
        _int8("prompt's fc1, 2309 tokens", 2309, 5120, 13824, gelu=True),
        # one token of a small vocabulary by its temperature alone: latency
        _sample("sample, one row", 1, 32000),
        # a batch's tree nodes, an odd vocabulary, top-k and top-p by row
        _sample("sample, 64 rows, k and p", 64, 100003, "f16", "kp"),
        # the largest: every filter, rows peaked and flat, by row
        _sample("sample, 256 rows, all filters", 256, 131072, "f32", "all"),
        # one sequence of a small decoder, one layer's cache: latency
        _accept("accept, one tree of 8", 1, 8, 1, 16, 64, 500),
        # a batch's trees, the caches of a decoder's layers
        _accept("accept, 16 trees, 24 layers", 16, 24, 24, 4, 128, 160),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["draft", "tree", "tree", "int8", "int8", "sample", "sample", "accept"])
    if kind == "draft":
        return dict(_draft("", _log(rng, 1, 64), _log(rng, 1, 64), _log(rng, 64, 8000)), kind=kind)
    if kind == "tree":
        D = rng.choice([64, 80, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
        B, nodes = _log(rng, 1, 32), _log(rng, 1, 100)
        longest = _log(rng, nodes, max(nodes + 1, min(65537, 2**26 // (B * kv_heads * D), 10**9 // (B * heads * nodes))))
        return _tree("", B, heads, kv_heads, D, longest, nodes)
    if kind == "int8":
        K = max(16, _log(rng, 64, 8192) // 16 * 16)
        N = max(4, _log(rng, 64, 65536) // 4 * 4)
        M = _log(rng, 1, max(1, min(4096, 10**11 // (K * N))))
        return _int8("", M, K, N, rng.random() < 0.5, rng.random() < 0.3, rng.choice(["f16", "f16", "f32"]), rng.choice(["f16", "f32"]))
    if kind == "sample":
        V = _log(rng, 100, 200000)
        return _sample("", _log(rng, 1, min(512, 2**25 // V)), V, rng.choice(["f16", "f32"]), rng.choice(["none", "k", "p", "min", "kp", "all", "all"]))
    B, D = _log(rng, 1, 32), rng.choice([64, 80, 128, 256])
    longest = _log(rng, 16, 400)
    kv_heads = rng.choice([1, 2, 4, 8])
    return _accept("", B, _log(rng, 1, min(64, longest)), max(1, min(_log(rng, 1, 32), 2**21 // (B * (longest + 128) * kv_heads * D // 64))), kv_heads, D, longest)


# ---- the cache's format ------------------------------------------------------------------------------------------------


def _padded(D):
    return 64 if D <= 64 else 128 if D <= 128 else 256


def _quantise(x, D):
    """x [..., D] fp32 -> codes [..., D] int32 in -7..7 and scales [..., ceil(D / 32)] fp16 of groups of 32 channels"""
    groups = -(-D // 32)
    g = torch.nn.functional.pad(x, (0, groups * 32 - D)).unflatten(-1, (groups, 32))
    u = (g.abs().amax(-1) * (1 / 7)).contiguous().view(torch.int32)
    u = ((u + 0xFFFF + ((u >> 17) & 1)) >> 17) << 17  # 7 significant bits
    s = u.view(torch.float32).to(torch.float16)
    s = torch.where(s == 0, torch.ones_like(s), s)
    c = torch.clamp(torch.round(g / s.float()[..., None]), -7, 7)
    return c.flatten(-2)[..., :D].to(torch.int32), s


def _pages(ck, sk, cv, sv, D):
    """Codes [pages, 64, heads, D] and scales [pages, 64, heads, groups] as cache pages [pages, heads, 72 * padded D]"""
    DP = _padded(D)
    J, CH = DP // 32, DP // 16
    pages, _, heads, _ = ck.shape
    pad = lambda c: torch.nn.functional.pad(c, (0, DP - D)).transpose(1, 2) + 8  # noqa: E731  [pages, heads, 64, DP]
    pads = lambda s: torch.nn.functional.pad(s, (0, J - s.shape[-1]), value=1.0).transpose(1, 2)  # noqa: E731
    # keys: word (g, j) of a token has channels 32 j + 8 g + 0..7, the even ones in its lower half
    k = pad(ck).view(pages, heads, _PAGE, J, 4, 4, 2).permute(0, 1, 2, 4, 3, 6, 5).to(torch.uint8)  # [.., g, j, parity, pair]
    k = (k[..., 0::2] | (k[..., 1::2] << 4)).reshape(pages, heads, -1)
    # values: quad of tokens, 16 blocks of CH channels, pair of tokens, four channels, token of the pair: 2 bytes
    v = pad(cv).view(pages, heads, _PAGE // 4, 2, 2, 16, CH // 4, 4).permute(0, 1, 2, 5, 3, 6, 4, 7).to(torch.uint8)
    v = (v[..., 0::2] | (v[..., 1::2] << 4)).reshape(pages, heads, -1)
    as_bytes = lambda s: s.contiguous().view(torch.uint8).reshape(pages, heads, -1)  # noqa: E731
    return torch.cat([k, as_bytes(pads(sk)), v, as_bytes(pads(sv).transpose(2, 3))], -1).contiguous()


def _cache_of_words(pages, D):
    """Pages [n, heads, bytes] as fp32 K, V [n, heads, 64, D]"""
    DP = _padded(D)
    J, CH = DP // 32, DP // 16
    n, heads, _ = pages.shape
    half, sc = 32 * DP, 128 * J
    four = 4 * torch.arange(4, device=pages.device, dtype=torch.int32)
    k = pages[..., :half].contiguous().view(torch.int16).view(n, heads, _PAGE, 4, J, 2, 1).to(torch.int32)
    k = ((k >> four) & 15).permute(0, 1, 2, 4, 3, 6, 5).reshape(n, heads, _PAGE, DP).float() - 8.0
    sk = pages[..., half:half + sc].contiguous().view(torch.float16).view(n, heads, _PAGE, J, 1).float()
    v = pages[..., half + sc:2 * half + sc].contiguous().view(torch.int16).view(n, heads, _PAGE // 4, 16, 2, CH // 4, 2, 1).to(torch.int32)
    v = ((v >> four) & 15).permute(0, 1, 2, 4, 6, 3, 5, 7).reshape(n, heads, _PAGE, DP).float() - 8.0
    sv = pages[..., 2 * half + sc:].contiguous().view(torch.float16).view(n, heads, J, _PAGE).transpose(2, 3)[..., None].float()
    K = (k.view(n, heads, _PAGE, J, 32) * sk).view(n, heads, _PAGE, DP)[..., :D]
    V = (v.view(n, heads, _PAGE, J, 32) * sv).view(n, heads, _PAGE, DP)[..., :D]
    return K, V


# ---- inputs ------------------------------------------------------------------------------------------------------------


def _counts(B, nodes):
    """Nodes of each sequence's tree: all of them, and fewer down to a half"""
    return [nodes - b * 5 % (nodes // 2 + 1) for b in range(B)]


def _follows(parents):
    """parents of one tree -> [n, n] bool: whether node i follows node j, or is it"""
    n = len(parents)
    f = np.eye(n, dtype=bool)
    for i, p in enumerate(parents):
        if p >= 0:
            f[i] |= f[p]
    return f


def _sequences(st, c, rng):
    """Ragged sequences with a tree each: counts, cu_q, lengths with the drafts, tables of pages"""
    B, L = c["B"], c["longest"]
    counts = _counts(B, c["nodes"])
    lens = [max(n, int(rng.integers(max(1, L // 4), L + 1))) for n in counts]
    lens[int(rng.integers(B))] = max(L, c["nodes"])
    if max(counts) < c["nodes"]:
        raise ValueError("no tree of all nodes")
    st["counts"], st["max_q"] = counts, c["nodes"]
    dev = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    st["cu_q"], st["lens"] = dev(np.cumsum([0] + counts)), dev(lens)
    per = -(-max(max(lens), 1) // _PAGE)
    used = [-(-n // _PAGE) for n in lens]
    total = B * per
    order, table, at = rng.permutation(total + 2), np.zeros((B, per), dtype=np.int32), 0
    for b in range(B):
        table[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
    st["block_table"], st["pages"] = dev(table), total + 2
    return dev, lens


def _cache(c, pages, gen):
    G, D = c["kv_heads"], c["D"]
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    cache, mean = torch.empty((pages, G, 72 * _padded(D)), dtype=torch.uint8, device="cuda"), 0.3 * normal(G, D)
    for a in range(0, pages, 256):
        n = min(256, pages - a)
        cache[a:a + n] = _pages(*_quantise(normal(n, _PAGE, G, D), D), *_quantise(normal(n, _PAGE, G, D) + mean, D), D)
    return cache


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=gen, device="cuda")  # noqa: E731
    c, st = case, dict(case=case)
    if c["kind"] in ("draft", "tree"):
        dev, _ = _sequences(st, c, rng)
        # node 0 is what was answered last; a draft follows any node in front of it, those right in front of it more often
        trees = [[-1] + [max(0, i - 1 - int(rng.integers(0, i) * rng.random())) for i in range(1, n)] for n in st["counts"]]
        st["parents"] = dev(sum(trees, []))
        if c["kind"] == "tree":
            W = -(-c["nodes"] // 32)
            rows = []
            for t in trees:
                f = np.zeros((len(t), 32 * W), dtype=np.uint8)
                f[:, :len(t)] = _follows(t)
                rows.append(np.packbits(f, axis=1, bitorder="little").view(np.int32))
            st["tree"] = dev(np.concatenate(rows))
            st["cache"] = _cache(c, st["pages"], gen)
            st["q"] = normal(len(st["parents"]), c["heads"], c["D"]).half() * 1.5
    elif c["kind"] == "int8":
        M, K, N = c["M"], c["K"], c["N"]
        # a few channels of the activations are larger than the others
        st["X"] = (normal(M, K) * (1 + 7 * (uniform(K) < 0.01))).to(_DT[c["x"]])
        st["Wq"] = torch.empty((N, K), dtype=torch.int8, device="cuda")
        for a in range(0, N, 16384):
            st["Wq"][a:a + 16384] = (normal(min(16384, N - a), K) * 32).round_().clamp_(-127, 127).to(torch.int8)
        st["w_scale"] = 0.02 / 32 * (0.7 + 0.6 * uniform(N))
        st["bias"] = 0.05 * normal(N) if c["bias"] else None
    elif c["kind"] == "sample":
        R, V, f = c["rows"], c["V"], c["filters"]
        x = 2.0 * normal(R, V)
        # rows with some likely tokens and flat ones, tokens that are never answered
        likely = torch.randint(V, (R, min(V, 24)), generator=gen, device="cuda")
        x.scatter_(1, likely, 4 + 9 * uniform(*likely.shape))
        x[2::3] *= 0.5
        x[:, V - V // 50:] = -math.inf
        st["x"], st["u"] = x.to(_DT[c["x"]]), uniform(R)
        pick = lambda values, dt: torch.tensor(values, dtype=dt, device="cuda")[torch.randint(len(values), (R,), generator=gen, device="cuda")].contiguous()  # noqa: E731
        st["T"] = pick([0.0, 0.6, 0.8, 1.0, 1.3], torch.float32)
        st["k"] = pick([0, 1, 20, 50, 1000], torch.int32) if f in ("k", "kp", "all") else None
        st["p"] = pick([0.5, 0.9, 0.95, 1.0], torch.float32) if f in ("p", "kp", "all") else None
        st["m"] = pick([0.0, 0.02, 0.1], torch.float32) if f in ("min", "all") else None
    else:
        dev, lens = _sequences(st, c, rng)
        parents, drafted, sampled = [], [], []
        for n in st["counts"]:
            # the branch that is kept: up to a third of the nodes, the rest of it drawn from those behind its own length, so that what is moved
            # is not what is written and a second pass over the same state moves the same
            want = int(rng.integers(0, (n - 1) // 2 + 1)) if n > 1 else 0
            want = min(want, 6)
            kept = [0] + sorted(int(v) for v in rng.choice(np.arange(want + 1, n), size=min(want, n - 1 - want), replace=False)) if want else [0]
            par, d, s = [-1] * n, [int(v) for v in rng.integers(0, 5, n)], [int(v) for v in rng.integers(5, 30000, n)]
            for i in range(1, n):
                par[i] = int(rng.integers(0, i))
            for a, b in zip(kept, kept[1:]):
                par[b], s[a] = a, 7 + a
                d[b] = s[a]
            parents += par
            drafted += d
            sampled += s
        st.update(parents=dev(parents), drafted=dev(drafted), sampled=dev(sampled))
        st["caches"] = [_cache(c, st["pages"], gen) for _ in range(c["layers"])]
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------------


def _run_own(st):
    from paper_2305_10727_amd import gpusq as G
    c = st["case"]
    if c["kind"] == "draft":
        return G.draft_tree(st["parents"], st["lens"], st["block_table"], cu_q=st["cu_q"], max_q=st["max_q"])
    if c["kind"] == "tree":
        return G.attention_kv4(st["q"], st["cache"], st["block_table"], st["lens"], cu_q=st["cu_q"], max_q=st["max_q"], tree=st["tree"])
    if c["kind"] == "int8":
        return G.linear_int8_tokens(st["X"], st["Wq"], st["w_scale"], bias=st["bias"], gelu=c["gelu"], out_dtype=_DT[c["out"]])
    if c["kind"] == "sample":
        return G.sample_tokens(st["x"], st["u"], temperature=st["T"], top_k=st["k"], top_p=st["p"], min_p=st["m"])
    path, accepted, answers, lens = G.accept_drafts(st["drafted"], st["sampled"], st["parents"], st["lens"], cu_q=st["cu_q"], max_q=st["max_q"],
                                                    caches=st["caches"], block_table=st["block_table"])
    return path, accepted, answers, lens, st["caches"]


def _padded_rows(st, x, fill):
    """x [tokens] of ragged sequences -> [B, max_q], and which are real"""
    cu, n = st["cu_q"].long(), st["max_q"]
    i = torch.arange(n, device="cuda")[None] + cu[:-1, None]
    real = i < cu[1:, None]
    return torch.where(real, x[i.clamp(max=len(x) - 1)].long(), torch.full_like(i, fill)), real


def _place_of(st, b, place):
    """Page and token of a place of sequence b"""
    return st["block_table"].long()[b, place // _PAGE], place % _PAGE


def _run_draft(st):
    parents, real = _padded_rows(st, st["parents"], -1)
    B, n = parents.shape
    follows = torch.eye(n, dtype=torch.bool, device="cuda").repeat(B, 1, 1)
    seq = torch.arange(B, device="cuda")
    for i in range(1, n):  # (a parent is in front of its node)
        p = parents[:, i]
        follows[:, i] |= follows[seq, p.clamp(min=0)] & (p >= 0)[:, None]
    W = -(-n // 32)
    bits = torch.nn.functional.pad(follows, (0, 32 * W - n)).view(B, n, W, 32).long()
    words = (bits << torch.arange(32, device="cuda")).sum(-1)
    words = torch.where(words >= 2**31, words - 2**32, words).to(torch.int32)
    before = st["lens"].long() - (st["cu_q"][1:] - st["cu_q"][:-1]).long()
    positions = before[:, None] + follows.sum(-1) - 1
    place = before[:, None] + torch.arange(n, device="cuda")[None]
    page, token = _place_of(st, seq[:, None], place.clamp(max=st["block_table"].shape[1] * _PAGE - 1))
    slots = page * _PAGE + token
    return words[real], positions[real].to(torch.int32), slots[real].to(torch.int32)


def _run_tree(st):
    c = st["case"]
    B, H, G, D = c["B"], c["heads"], c["kv_heads"], c["D"]
    rep = H // G
    K, V = _cache_of_words(st["cache"], D)
    per = st["block_table"].shape[1]
    at = st["block_table"].long().reshape(-1)
    K, V = (x[at].view(B, per, G, _PAGE, D).transpose(1, 2).reshape(B, G, per * _PAGE, D) for x in (K, V))
    cu, lens, new = st["cu_q"].long(), st["lens"].long(), st["max_q"]
    i = torch.arange(new, device="cuda")[None] + cu[:-1, None]
    real = i < cu[1:, None]
    i = i.clamp(max=st["q"].shape[0] - 1)
    q = st["q"].float()[i].view(B, new, G, rep, D).permute(0, 2, 1, 3, 4).reshape(B, G, new * rep, D)
    before = (lens - (cu[1:] - cu[:-1]))[:, None, None]
    node = torch.arange(per * _PAGE, device="cuda")[None, None] - before  # [B, 1, S]
    words = st["tree"].long()[i]  # [B, new, W]
    inside = (node >= 0) & (node < (cu[1:] - cu[:-1])[:, None, None])
    bit = (torch.gather(words, 2, (node.clamp(0, 32 * words.shape[2] - 1) // 32).expand(B, new, -1)) >> (node.clamp(min=0) % 32)) & 1
    visible = ((node < 0) | (inside & (bit != 0))) & real[..., None]
    visible = visible.repeat_interleave(rep, 1)[:, None]
    s = torch.matmul(q, K.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    s = torch.where(visible, s, torch.full_like(s[:1, :1, :1, :1], -math.inf))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, V) / torch.where(total == 0, torch.ones_like(total), total)
    return o.view(B, G, new, rep, D).permute(0, 2, 1, 3, 4).reshape(B, new, H, D)[real].half()


def _run_int8(st):
    c = st["case"]
    x = st["X"].float()
    most = x.abs().amax(1, keepdim=True)
    s = most / torch.full_like(most, 127.0)  # (by a plain number torch multiplies with its reciprocal)
    s = torch.where(s == 0, torch.ones_like(s), s)
    q = torch.clamp(torch.round(x / s), -127, 127)
    y = torch.matmul(q, st["Wq"].float().t()) * s * st["w_scale"]
    y = y if st["bias"] is None else y + st["bias"]
    y = 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0))) if c["gelu"] else y
    return y.to(_DT[c["out"]])


def _run_sample(st):
    x = st["x"].double()
    R, V = x.shape
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    x, order = torch.sort(x, dim=1, descending=True, stable=True)  # (ties: the lowest index first)
    T = st["T"].double()[:, None]
    top = x[:, :1]
    w = torch.exp((x - top) / torch.where(T > 0, T, torch.ones_like(T)))
    w = torch.where(x == top, torch.ones_like(w), torch.where(w < _LEAST, torch.zeros_like(w), w))
    w = torch.where(top == -math.inf, torch.zeros_like(w), w)
    rank = torch.arange(V, device="cuda")[None]
    keep = (T > 0) | (rank == 0)
    if st["k"] is not None:
        keep = keep & ((st["k"][:, None] <= 0) | (rank < st["k"][:, None]))
    w = torch.where(keep, w, torch.zeros_like(w))
    if st["p"] is not None:
        p = st["p"].double()[:, None]
        before = torch.cumsum(w, 1) - w
        w_p = torch.where((before < p * w.sum(1, keepdim=True)) | (p >= 1) | (rank == 0), w, torch.zeros_like(w))
    else:
        w_p = w
    if st["m"] is not None:
        w_p = torch.where(w_p >= st["m"].double()[:, None].clamp(max=1.0), w_p, torch.zeros_like(w))
    w = torch.empty_like(w_p).scatter_(1, order, w_p)  # by the vocabulary's order again
    upto = torch.cumsum(w, 1)
    total = upto[:, -1:]
    token = (upto <= st["u"].double()[:, None] * total).sum(1, keepdim=True).clamp(max=V - 1)
    some = total > 0
    prob = torch.where(some, torch.gather(w, 1, token) / torch.where(some, total, torch.ones_like(total)), torch.zeros_like(total))
    return torch.where(some, token, torch.full_like(token, -1))[:, 0].to(torch.int32), prob[:, 0].float()


def _run_accept(st):
    parents, real = _padded_rows(st, st["parents"], -1)
    drafted, _ = _padded_rows(st, st["drafted"], -1)
    sampled, _ = _padded_rows(st, st["sampled"], -2)
    B, n = parents.shape
    seq = torch.arange(B, device="cuda")
    at, path = torch.zeros(B, dtype=torch.long, device="cuda"), torch.full((B, n), -1, device="cuda")
    path[:, 0] = 0
    on = torch.ones(B, dtype=torch.bool, device="cuda")
    node = torch.arange(n, device="cuda")[None]
    for i in range(1, n):
        fits = real & (parents == at[:, None]) & (drafted == sampled[seq, at][:, None]) & (node > at[:, None])
        on = on & fits.any(1)
        at = torch.where(on, fits.long().argmax(1), at)
        path[:, i] = torch.where(on, at, torch.full_like(at, -1))
    accepted = (path >= 0).sum(1)
    before = st["lens"].long() - (st["cu_q"][1:] - st["cu_q"][:-1]).long()
    # what is kept moves together: all of it is read, then written
    b, i = torch.nonzero(path > 0, as_tuple=True)
    (p0, t0), (p1, t1) = _place_of(st, b, before[b] + path[b, i]), _place_of(st, b, before[b] + i)
    D = st["case"]["D"]
    DP = _padded(D)
    J = DP // 32
    for cache in st["caches"]:
        pages, G, _ = cache.shape
        k, ks = cache[..., :32 * DP].view(pages, G, _PAGE, DP // 2), cache[..., 32 * DP:36 * DP].view(pages, G, _PAGE, 2 * J)
        v = cache[..., 36 * DP:68 * DP].view(pages, G, _PAGE // 4, 16, 2, DP // 64, 2, 2)  # quad, channels, pair, channels, token, bytes
        vs = cache[..., 68 * DP:].view(pages, G, J, _PAGE, 2)
        moved = [x[p0, :, t0] for x in (k, ks)] + [v[p0, :, t0 // 4, :, t0 % 4 // 2, :, t0 % 2], vs[p0, :, :, t0]]
        k[p1, :, t1], ks[p1, :, t1] = moved[0], moved[1]
        v[p1, :, t1 // 4, :, t1 % 4 // 2, :, t1 % 2], vs[p1, :, :, t1] = moved[2], moved[3]
    i32 = torch.int32
    return path.to(i32), accepted.to(i32), sampled[seq, at].to(i32), (before + accepted).to(i32), st["caches"]


def _run_plain(st):
    return dict(draft=_run_draft, tree=_run_tree, int8=_run_int8, sample=_run_sample, accept=_run_accept)[st["case"]["kind"]](st)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------


def work(case):
    c = case
    if c["kind"] in ("draft", "tree", "accept"):
        counts = _counts(c["B"], c["nodes"])
        tokens, words = sum(counts), -(-c["nodes"] // 32)
    if c["kind"] == "draft":
        return {"bytes": tokens * (4 + 4 * words + 8 + 4) + 8.0 * c["B"], "flops": 1.0 * sum(n * n for n in counts)}
    if c["kind"] == "tree":
        # (lengths are even over a quarter of the longest to all of it)
        H, G, D = c["heads"], c["kv_heads"], c["D"]
        kept = max(c["longest"], c["nodes"]) * (1 + 0.625 * (c["B"] - 1))
        return {"bytes": kept * G * D * 2 * 0.5625 + 4.0 * tokens * H * D + 4.0 * tokens * words, "flops": 4.0 * tokens * H * D * max(1.0, kept / c["B"])}
    if c["kind"] == "int8":
        M, K, N = c["M"], c["K"], c["N"]
        return {"bytes": 1.0 * N * K + (4 if c["x"] == "f32" else 2) * M * K + (4 if c["out"] == "f32" else 2) * M * N + (8 if c["bias"] else 4) * N, "flops": 2.0 * M * N * K}
    if c["kind"] == "sample":
        return {"bytes": c["rows"] * (c["V"] * (4.0 if c["x"] == "f32" else 2.0) + 28), "flops": 8.0 * c["rows"] * c["V"]}
    moved = 1.5 * c["B"] * min(1.0, c["nodes"] / 8)  # (about)
    return {"bytes": 12.0 * tokens + 4.0 * c["B"] * (c["nodes"] + 5) + 2 * 2 * 0.5625 * moved * c["layers"] * c["kv_heads"] * c["D"], "flops": 2.0 * tokens}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def _exact_cache(pages, D):
    DP = _padded(D)
    J, CH = DP // 32, DP // 16
    t, d = torch.arange(_PAGE, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    at_k = t * DP // 2 + (d % 32 // 8 * J + d // 32) * 4 + d % 2 * 2 + d % 8 // 4
    at_v = 32 * DP + 128 * J + ((t // 4 * 16 + d // CH) * 2 + t % 4 // 2) * CH + d % CH // 4 * 4 + t % 2 * 2 + d % 4 // 2
    halves = pages.view(torch.float16)
    K = ((pages[..., at_k].int() >> (d % 8 // 2 % 2 * 4)) & 15).double() - 8
    V = ((pages[..., at_v].int() >> (d % 2 * 4)) & 15).double() - 8
    return K * halves[..., 16 * DP + t * J + d // 32].double(), V * halves[..., 32 * DP + 64 * J + d // 32 * _PAGE + t].double()


def _exact_row(x, u, T, k, p, m):
    """One row of logits (numpy, 64 bits) -> token, probability"""
    x = np.where(np.isnan(x), -np.inf, x)
    V = len(x)
    top = x.max()
    if top == -np.inf:
        return -1, 0.0
    if not T > 0:
        return int(np.argmax(x)), 1.0
    with np.errstate(invalid="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / T))
    w[w < _LEAST] = 0.0
    order = np.lexsort((np.arange(V), -x))  # by value, then by index
    n = V if k <= 0 else min(k, V)
    mass = np.cumsum(w[order[:n]])
    if p < 1:
        n = max(1, min(n, int(np.searchsorted(mass, p * mass[-1], side="left")) + 1))
    kept = np.zeros(V, dtype=bool)
    kept[order[:n]] = True
    w = np.where(kept & (w >= min(m, 1.0)), w, 0.0)
    upto = np.cumsum(w)
    token = min(int(np.searchsorted(upto, u * upto[-1], side="right")), V - 1)
    return token, w[token] / upto[-1]


def exact(case, seed):
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] in ("draft", "tree"):
        cu, lens, table = st["cu_q"].tolist(), st["lens"].tolist(), st["block_table"].cpu().numpy()
        W = -(-c["nodes"] // 32)
        parents = st["parents"].tolist()
        outs = []
        for b in range(c["B"]):
            n, t = cu[b + 1] - cu[b], parents[cu[b]:cu[b + 1]]
            chains = []  # the nodes that each one follows, itself among them
            for i in range(n):
                chain = [i]
                while t[chain[-1]] >= 0:
                    chain.append(t[chain[-1]])
                chains.append(chain)
            if c["kind"] == "draft":
                words = np.zeros((n, W), dtype=np.uint32)
                for i, chain in enumerate(chains):
                    for j in chain:
                        words[i, j // 32] |= np.uint32(1) << np.uint32(j % 32)
                place = [lens[b] - n + i for i in range(n)]
                outs.append((words.view(np.int32), np.array([lens[b] - n + len(x) - 1 for x in chains]), np.array([table[b, q // _PAGE] * _PAGE + q % _PAGE for q in place])))
                continue
            K, V = _exact_cache(st["cache"][st["block_table"].long()[b, :-(-lens[b] // _PAGE)]], c["D"])
            K, V = (x.transpose(0, 1).reshape(c["kv_heads"], -1, c["D"])[:, :lens[b]] for x in (K, V))
            seen = torch.zeros((n, lens[b]), dtype=torch.bool)
            seen[:, :lens[b] - n] = True
            for i, chain in enumerate(chains):
                seen[i, [lens[b] - n + j for j in chain]] = True
            seen, q = seen.cuda(), st["q"][cu[b]:cu[b + 1]].to(f64)
            heads = []
            for h in range(c["heads"]):
                s = q[:, h] @ K[h * c["kv_heads"] // c["heads"]].t() / c["D"] ** 0.5
                heads.append(torch.softmax(s.masked_fill(~seen, -math.inf), 1) @ V[h * c["kv_heads"] // c["heads"]])
            outs.append(torch.stack(heads, 1))
        if c["kind"] == "tree":
            return torch.cat(outs)
        return tuple(torch.tensor(np.concatenate(x), dtype=torch.int32) for x in zip(*outs))
    if c["kind"] == "int8":
        ys, x = [], st["X"].to(f64)
        s = (x.abs().amax(1) / 127).float()  # a scale is 32 bits, and so is a quotient (of 64 bits rounded once more it is the same)
        s = torch.where(s == 0, torch.ones_like(s), s).to(f64)[:, None]
        q = (x / s).float().to(f64).round().clamp(-127, 127)
        for a in range(0, c["N"], 8192):
            ys.append(q @ st["Wq"][a:a + 8192].to(f64).t())
        y = torch.cat(ys, 1) * s * st["w_scale"].to(f64) + (0 if st["bias"] is None else st["bias"].to(f64))
        return y * torch.special.ndtr(y) if c["gelu"] else y
    if c["kind"] == "sample":
        x, R = st["x"].double().cpu().numpy(), c["rows"]
        col = lambda t, none: [none] * R if t is None else t.double().tolist()  # noqa: E731
        got = [_exact_row(*a) for a in zip(x, col(st["u"], 0), col(st["T"], 1), [int(k) for k in col(st["k"], 0)], col(st["p"], 1.0), col(st["m"], 0.0))]
        return torch.tensor([t for t, _ in got], dtype=torch.int32), torch.tensor([p for _, p in got], dtype=f64)
    # accept: the formats' places one by one, in bytes
    cu, lens, table = st["cu_q"].tolist(), st["lens"].tolist(), st["block_table"].tolist()
    caches = [x.cpu().numpy() for x in st["caches"]]
    DP = _padded(c["D"])
    J, CH = DP // 32, DP // 16
    ch = np.arange(DP // 4)  # quads of channels: 16 blocks of CH / 4
    bits = lambda t: np.concatenate([  # noqa: E731  the bytes of token t of a head's page
        np.arange(t * DP // 2, (t + 1) * DP // 2), 32 * DP + np.arange(t * 2 * J, (t + 1) * 2 * J),
        36 * DP + (2 * ((((t // 4 * 16 + ch // (CH // 4)) * 2 + t % 4 // 2) * (DP // 64) + ch % (CH // 4)) * 2 + t % 2)[:, None] + np.arange(2)).ravel(),
        68 * DP + (2 * (np.arange(J) * _PAGE + t)[:, None] + np.arange(2)).ravel()])
    path, accepted, answers, new = np.full((c["B"], c["nodes"]), -1), [], [], []
    for b in range(c["B"]):
        n = cu[b + 1] - cu[b]
        par, d, s = (st[k].tolist()[cu[b]:cu[b + 1]] for k in ("parents", "drafted", "sampled"))
        kept = [0]
        while True:
            follow = [i for i in range(kept[-1] + 1, n) if par[i] == kept[-1] and d[i] == s[kept[-1]]]
            if not follow:
                break
            kept.append(follow[0])
        path[b, :len(kept)] = kept
        accepted.append(len(kept))
        answers.append(s[kept[-1]])
        new.append(lens[b] - n + len(kept))
        for i, j in enumerate(kept):  # in order: what is written is in front of all that is still to be read
            to, at = lens[b] - n + i, lens[b] - n + j
            for x in caches:
                x[table[b][to // _PAGE]][:, bits(to % _PAGE)] = x[table[b][at // _PAGE]][:, bits(at % _PAGE)]
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32)  # noqa: E731
    return i32(path), i32(accepted), i32(answers), i32(new), [torch.from_numpy(x) for x in caches]
