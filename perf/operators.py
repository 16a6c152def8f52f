"""Timed cases of the operators of a decoder that answers from what an encoder has seen, one pass of one operator each.

Kinds of case
  linear  a linear layer on 4-bit weights with group scales for a few tokens (`gpusq.linear_int4`)
  rope    the norms of queries and keys per head and the position rotation, from a packed projection (`gpusq.qk_norm_rope`);
          with `cache` the keys and values go into the 4-bit cache in the same pass, and come back as what the cache stands for
  self    attention over the paged 4-bit cache (`gpusq.attention_kv4`): one new token a sequence, or a ragged chunk of new ones
  cross   attention to an encoder's states of another length (`gpusq.cross_attention`), or of the same length: the encoder's own

The plain forms compute in 32 bits and round once at the end.  exact() is the definition in 64 bits; it finds codes and scales by
their places in the formats of include/gpusq.h one by one, where the plain forms unpack whole words.
"""
import math

import torch

own = False

_DT = {"f16": torch.float16, "f32": torch.float32}
_PAGE = 64  # tokens of a page of the cache


def _linear(name, M, K, N, group, bias=True, gelu=False, out="f16"):
    return dict(name=name, kind="linear", M=M, K=K, N=N, group=group, bias=bias, gelu=gelu, out=out)


def _rope(name, T, heads, kv_heads, D, R, table, interleaved=False, norm=True, cache=False, x="f16"):
    return dict(name=name, kind="rope", T=T, heads=heads, kv_heads=kv_heads, D=D, R=R, table=table, interleaved=interleaved, norm=norm, cache=cache, x=x)


def _self(name, B, heads, kv_heads, D, longest, new=1):
    return dict(name=name, kind="self", B=B, heads=heads, kv_heads=kv_heads, D=D, longest=longest, new=new)


def _cross(name, B, Tq, S, heads, kv_heads, D, mask="none", packed=False):
    return dict(name=name, kind="cross", B=B, Tq=Tq, S=S, heads=heads, kv_heads=kv_heads, D=D, mask=mask, packed=packed)


def listed():
    return [
        # one token through a small layer: the launch and the latency of memory
        _linear("4-bit layer, one token", 1, 1024, 1024, 32),
        # one token through a feed-forward layer with GELU: the weights' bytes
        _linear("4-bit fc1, one token", 1, 5120, 13824, 128, gelu=True),
        # an odd number of tokens (speculated ones, a small batch) through the largest layer, 4-byte output
        _linear("4-bit wide layer, 13 tokens", 13, 8192, 24576, 64, bias=False, out="f32"),
        # one token of a small decoder: queries, keys and values of 16 heads, into the cache
        _rope("norm and rotation, one token", 1, 16, 16, 64, 64, 2048, cache=True),
        # a prompt's chunk of 509 tokens with grouped heads, into the cache
        _rope("norm and rotation, 509 tokens", 509, 32, 8, 128, 128, 8192, cache=True),
        # ViT-H/14 at batch 128: the queries and keys of every image, rotated by the patch's place, heads of 80
        _rope("norm and rotation, ViT-H images", 128 * 257, 16, 16, 80, 80, 257, interleaved=True),
        # one sequence with a long history: the work has to be split over it
        _self("cache, one long sequence", 1, 32, 8, 128, 131071),
        # a serving batch of ragged lengths
        _self("cache, 64 ragged sequences", 64, 32, 8, 128, 4096),
        # chunks of prompts behind a history: many rows for one pass over the cache
        _self("cache, chunks of 300", 2, 32, 8, 128, 6000, new=300),
        # one token that looks at one image (ViT-H/14: 257 states, heads of 80)
        _cross("one token to one image", 1, 1, 257, 16, 16, 80),
        # the encoder's own attention, ViT-B at batch 128, from the packed projection
        _cross("ViT-B attention", 128, 197, 197, 12, 12, 64, packed=True),
        # prompts that look at several images each, ragged, grouped heads
        _cross("prompts to images, ragged", 4, 1000, 2313, 32, 8, 128, mask="lens"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "rope", "self", "cross"])
    if kind == "linear":
        group = rng.choice([32, 64, 128])
        K = max(group, _log(rng, 256, 8192) // group * group)
        return dict(_linear("", _log(rng, 1, 64), K, max(1, _log(rng, 256, 24576) // 4) * 4, group, rng.random() < 0.5, rng.random() < 0.3, rng.choice(["f16", "f16", "f32"])), kind=kind)
    if kind == "rope":
        D = rng.choice([64, 64, 80, 96, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
        cache = rng.random() < 0.6
        most = 2**19 // (kv_heads * D) if cache else min(40000, 10**8 // ((heads + 2 * kv_heads) * D))
        R = rng.choice([D, D, D // 32 * 16])
        return _rope("", _log(rng, 1, most), heads, kv_heads, D, R, _log(rng, 64, 8192), rng.random() < 0.4, rng.random() < 0.8, cache, rng.choice(["f16", "f16", "f32"]))
    if kind == "self":
        D = rng.choice([64, 80, 128, 128, 256])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
        B = _log(rng, 1, 64)
        longest = _log(rng, 1, min(131071, 2**28 // (B * kv_heads * D)))
        new = 1
        if rng.random() < 0.3:
            new = min(longest, max(1, _log(rng, 2, min(300, 1 + 3 * 10**8 // (B * heads * longest)))))
        return _self("", B, heads, kv_heads, D, longest, new)
    D = rng.choice([64, 64, 80, 96, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 12, 16])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4])
    S = _log(rng, 1, 4096)
    Tq = S if rng.random() < 0.2 else rng.choice([1, _log(rng, 1, 1500)])
    Tq = max(1, min(Tq, 18 * 10**7 // (heads * S)))
    B = max(1, min(_log(rng, 1, 128), 18 * 10**7 // (heads * S * Tq), 10**8 // (kv_heads * S * D)))
    packed = Tq == S
    return _cross("", B, Tq, S, heads, kv_heads, D, rng.choice(["none", "lens", "bytes"]), packed)


# ---- the formats -------------------------------------------------------------------------------------------------------


def _padded(D):
    return 64 if D <= 64 else 128 if D <= 128 else 256


def _round7(s):
    """fp32 to 7 significant bits, half to even, held as fp16 in 2^-24 .. 896 (what rounds to 0: 1)"""
    u = s.contiguous().view(torch.int32)
    u = ((u + 0xFFFF + ((u >> 17) & 1)) >> 17) << 17
    s = torch.minimum(u.view(torch.float32), torch.full_like(s, 896.0)).to(torch.float16)
    return torch.where(s == 0, torch.ones_like(s), s)


def _quantise(x, D):
    """x [..., D] fp32 -> codes [..., D] int32 in -7..7 and scales [..., ceil(D / 32)] fp16 of groups of 32 channels"""
    groups = -(-D // 32)
    g = torch.nn.functional.pad(x, (0, groups * 32 - D)).unflatten(-1, (groups, 32))
    most = g.abs().amax(-1)
    s = _round7(most / torch.full_like(most, 7.0))  # (by a plain number torch multiplies with its reciprocal, and quotients that are ties are common)
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
    k = pad(ck).view(pages, heads, _PAGE, J, 4, 4, 2).permute(0, 1, 2, 4, 3, 6, 5)  # [.., g, j, parity, pair]
    k = (k.to(torch.uint8)[..., 0::2] | (k.to(torch.uint8)[..., 1::2] << 4)).reshape(pages, heads, -1)
    # values: quad of tokens, 16 blocks of CH channels, pair of tokens, four channels, token of the pair: 2 bytes
    v = pad(cv).view(pages, heads, _PAGE // 4, 2, 2, 16, CH // 4, 4).permute(0, 1, 2, 5, 3, 6, 4, 7)
    v = (v.to(torch.uint8)[..., 0::2] | (v.to(torch.uint8)[..., 1::2] << 4)).reshape(pages, heads, -1)
    as_bytes = lambda s: s.contiguous().view(torch.uint8).reshape(pages, heads, -1)  # noqa: E731
    return torch.cat([k, as_bytes(pads(sk)), v, as_bytes(pads(sv).transpose(2, 3))], -1).contiguous()


def _pack_weights(codes, scales, group):
    """codes [N, K] int8, scales [N, K / group] fp16 -> the packed operand of linear_int4 (uint8)"""
    N, K = codes.shape
    nt, kt = -(-N // 16), -(-K // 128)
    c = torch.nn.functional.pad(codes, (0, kt * 128 - K, 0, nt * 16 - N)) + 8
    # step, row of 16: word (j) of lane (g, r) has k = 32 j + 8 g + 0..7, the even ones in its lower half
    c = c.view(nt, 16, kt, 4, 4, 4, 2).permute(0, 2, 4, 1, 3, 6, 5).to(torch.uint8)  # [nt, kt, g, r, j, parity, pair]
    c = (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(-1)
    s = torch.nn.functional.pad(scales, (0, kt * (128 // group) - K // group, 0, nt * 16 - N))
    s = s.view(nt, 16, kt * (128 // group)).permute(0, 2, 1).contiguous().view(torch.uint8).reshape(-1)
    return torch.cat([c, s])


def _weights_of_words(packed, N, K, group):
    """The packed operand as fp32 [N, K]"""
    nt, kt = -(-N // 16), -(-K // 128)
    cut = nt * kt * 1024
    w = packed[:cut].view(torch.int32).view(nt, kt, 4, 16, 4, 1)
    c = ((w >> (4 * torch.arange(8, device=w.device, dtype=torch.int32))) & 15).to(torch.int8)
    c = c.view(nt, kt, 4, 16, 4, 2, 4).permute(0, 3, 1, 4, 2, 6, 5).reshape(nt * 16, kt * 128)[:N, :K]
    s = packed[cut:].view(torch.float16).view(nt, -1, 16).permute(0, 2, 1).reshape(nt * 16, -1)[:N, :K // group]
    return ((c.float() - 8.0).view(N, K // group, group) * s.float()[..., None]).view(N, K)


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


def _table(rows, R):
    """cos and sin [rows, R / 2] of the usual frequencies"""
    f = 10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / max(R, 1))
    a = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    whole = lambda hi, *shape, lo=0: torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)  # noqa: E731
    c, st = case, dict(case=case)
    if c["kind"] == "linear":
        M, K, N, group = c["M"], c["K"], c["N"], c["group"]
        scale = 0.02 / 2.5 * (0.7 + 0.6 * torch.rand((N, K // group), generator=gen, device="cuda"))
        codes = torch.empty((N, K), dtype=torch.int8, device="cuda")
        for a in range(0, N, 4096):  # (by rows: the normal numbers of the largest layer are a gigabyte)
            codes[a:a + 4096] = (normal(min(4096, N - a), K) * 2.5).round_().clamp_(-7, 7).to(torch.int8)
        st.update(X=normal(M, K).half(), packed=_pack_weights(codes, scale.half(), group), bias=normal(N) * 0.01 if c["bias"] else None)
    elif c["kind"] == "rope":
        T, H, G, D, R = c["T"], c["heads"], c["kv_heads"], c["D"], c["R"]
        st["qkv"] = (normal(T, (H + 2 * G) * D) * 1.2).to(_DT[c["x"]])
        st["qw"], st["kw"] = (1 + 0.1 * normal(D), 1 + 0.1 * normal(D)) if c["norm"] else (None, None)
        st["cos"], st["sin"] = _table(c["table"], R)
        start = int(whole(max(1, c["table"] - T + 1), 1)) if T <= c["table"] else 0
        st["positions"] = ((torch.arange(T, device="cuda", dtype=torch.int32) + start) % c["table"]).to(torch.int32)
        if c["cache"]:
            pages = -(-T // _PAGE) + 3
            st["cache"] = torch.zeros((pages, G, 72 * _padded(D)), dtype=torch.uint8, device="cuda")
            order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
            at = torch.arange(T, device="cuda", dtype=torch.int32) + 37  # (the chunk begins inside a page)
            st["slots"] = order[(at // _PAGE).long()] * _PAGE + at % _PAGE
    elif c["kind"] == "self":
        B, H, G, D, L = c["B"], c["heads"], c["kv_heads"], c["D"], c["longest"]
        # new tokens: all of them, and fewer down to a half; lengths: the longest, and fewer down to a quarter
        new = c["new"] - torch.arange(B, device="cuda", dtype=torch.int32) * 37 % (c["new"] // 2 + 1)
        lens = torch.maximum(whole(L + 1, B, lo=max(1, L // 4)), new)
        lens[int(whole(B, 1))] = L
        per = -(-L // _PAGE)
        used = (lens + _PAGE - 1) // _PAGE
        total = int(used.sum())
        order = torch.randperm(total + 2, generator=gen, device="cuda").to(torch.int32)
        first = torch.cumsum(used, 0) - used
        i = torch.arange(per, device="cuda")[None] + first[:, None]
        st["block_table"] = torch.where(torch.arange(per, device="cuda")[None] < used[:, None], order[i.clamp(max=total + 1)], torch.zeros_like(order[:1])).to(torch.int32).contiguous()
        st["cache"] = torch.empty((total + 2, G, 72 * _padded(D)), dtype=torch.uint8, device="cuda")
        mean = 0.3 * normal(G, D)
        for a in range(0, total + 2, 256):
            n = min(256, total + 2 - a)
            k, v = _quantise(normal(n, _PAGE, G, D), D), _quantise(normal(n, _PAGE, G, D) + mean, D)
            st["cache"][a:a + n] = _pages(*k, *v, D)
        st["cu_q"] = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0)).to(torch.int32)
        st["max_q"], st["lens"], st["q"] = int(new.max()), lens, normal(int(new.sum()), H, D).half() * 1.5
    else:
        B, Tq, S, H, G, D = c["B"], c["Tq"], c["S"], c["heads"], c["kv_heads"], c["D"]
        if c["packed"]:  # one projection's output, looked at where it is
            qkv = normal(B, S, H + 2 * G, D).half()
            st["q"], st["k"], st["v"] = qkv[:, :, :H], qkv[:, :, H:H + G], qkv[:, :, H + G:]
        else:
            st["q"], st["k"], st["v"] = normal(B, Tq, H, D).half() * 1.5, normal(B, S, G, D).half(), (normal(B, S, G, D) + 0.3 * normal(G, D)).half()
        st["lens"] = whole(S + 1, B, lo=S // 2) if c["mask"] == "lens" else None
        st["mask"] = (torch.rand((B, S), generator=gen, device="cuda") < 0.8).to(torch.uint8) if c["mask"] == "bytes" else None
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------------


def _run_own(st):
    from paper_2305_10727_amd import gpusq as G
    c = st["case"]
    if c["kind"] == "linear":
        return G.linear_int4(st["X"], st["packed"], c["N"], c["group"], bias=st["bias"], gelu=c["gelu"], out_dtype=_DT[c["out"]])
    if c["kind"] == "rope":
        sizes = (c["heads"], c["kv_heads"], c["D"])
        how = dict(q_weight=st["qw"], k_weight=st["kw"], eps=1e-6, norm=c["norm"], cos=st["cos"], sin=st["sin"], positions=st["positions"], interleaved=c["interleaved"])
        if c["cache"]:
            return G.qk_norm_rope(st["qkv"], *sizes, **how, cache=st["cache"], slots=st["slots"], want_cached=True)
        return G.qk_norm_rope(st["qkv"], *sizes, **how)
    if c["kind"] == "self":
        return G.attention_kv4(st["q"], st["cache"], st["block_table"], st["lens"], cu_q=st["cu_q"] if c["new"] > 1 else None, max_q=st["max_q"])
    return G.cross_attention(st["q"], st["k"], st["v"], kv_lens=st["lens"], key_mask=st["mask"])


def _normed(x, weight):
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    return y if weight is None else y * weight


def _rotated(x, cos, sin, R, interleaved):
    """x [T, heads, D]; cos, sin [T, 1, R / 2]"""
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((y, x[..., R:]), -1)


def _attend(q, k, v, visible):
    """q [B, G, rows, D], k, v [B, G, S, D] fp32, visible [B, 1 or G, 1 or rows, S]: a row that sees nothing gives 0"""
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(q.shape[-1]))
    s = torch.where(visible, s, torch.full_like(s[:1, :1, :1, :1], -math.inf))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)


def _run_plain(st):
    c = st["case"]
    if c["kind"] == "linear":
        y = torch.matmul(st["X"].float(), _weights_of_words(st["packed"], c["N"], c["K"], c["group"]).t())
        y = y if st["bias"] is None else y + st["bias"]
        y = 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0))) if c["gelu"] else y
        return y.to(_DT[c["out"]])
    H, G, D = c["heads"], c["kv_heads"], c["D"]
    if c["kind"] == "rope":
        x = st["qkv"].float().view(c["T"], H + 2 * G, D)
        q, k, v = x[:, :H], x[:, H:H + G], x[:, H + G:]
        if c["norm"]:
            q, k = _normed(q, st["qw"]), _normed(k, st["kw"])
        at = st["positions"].long()
        cos, sin = st["cos"][at][:, None], st["sin"][at][:, None]
        q, k = _rotated(q, cos, sin, c["R"], c["interleaved"]), _rotated(k, cos, sin, c["R"], c["interleaved"])
        if not c["cache"]:
            return q.half(), k.half()
        held = lambda y: (y[0].float() * y[1].float().repeat_interleave(32, -1)[..., :D]).half()  # noqa: E731
        return q.half(), held(_quantise(k, D)), held(_quantise(v, D))
    if c["kind"] == "self":
        B, L, rep = c["B"], c["longest"], H // G
        K, V = _cache_of_words(st["cache"], D)
        per = st["block_table"].shape[1]
        at = st["block_table"].long().reshape(-1)
        K, V = (x[at].view(B, per, G, _PAGE, D).transpose(1, 2).reshape(B, G, per * _PAGE, D) for x in (K, V))
        new = st["max_q"]
        cu, lens = st["cu_q"].long(), st["lens"].long()
        i = torch.arange(new, device="cuda")[None] + cu[:-1, None]  # [B, new]
        real = i < cu[1:, None]
        q = st["q"].float()[i.clamp(max=st["q"].shape[0] - 1)]  # [B, new, H, D]
        q = q.view(B, new, G, rep, D).permute(0, 2, 1, 3, 4).reshape(B, G, new * rep, D)
        place = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + torch.arange(new, device="cuda")[None]
        visible = (torch.arange(per * _PAGE, device="cuda")[None, None] <= place[..., None]) & real[..., None]
        o = _attend(q, K, V, visible.repeat_interleave(rep, 1)[:, None])
        o = o.view(B, G, new, rep, D).permute(0, 2, 1, 3, 4).reshape(B, new, H, D)
        return o[real].half()
    B, Tq, S, rep = c["B"], c["Tq"], c["S"], H // G
    q = st["q"].float().view(B, Tq, G, rep, D).permute(0, 2, 1, 3, 4).reshape(B, G, Tq * rep, D)
    k, v = st["k"].float().transpose(1, 2).contiguous(), st["v"].float().transpose(1, 2).contiguous()
    visible = torch.ones((B, S), dtype=torch.bool, device="cuda")
    if st["lens"] is not None:
        visible = torch.arange(S, device="cuda")[None] < st["lens"][:, None]
    if st["mask"] is not None:
        visible = visible & (st["mask"] != 0)
    o = _attend(q, k, v, visible[:, None, None])
    return o.view(B, G, Tq, rep, D).permute(0, 2, 1, 3, 4).reshape(B, Tq, H, D).half()


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------


def work(case):
    c = case
    if c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        return {"bytes": N * K / 2 + 2 * N * K / c["group"] + 2 * M * K + (4 if c["out"] == "f32" else 2) * M * N + (4 * N if c["bias"] else 0), "flops": 2.0 * M * N * K}
    H, G, D = c["heads"], c["kv_heads"], c["D"]
    if c["kind"] == "rope":
        T, size = c["T"], 4 if c["x"] == "f32" else 2
        table = min(T, c["table"]) * c["R"] * 4
        if c["cache"]:
            return {"bytes": T * D * (size * (H + 2 * G) + 2 * H + 2 * G * (2 + 0.5625)) + table, "flops": 10.0 * T * (H + 2 * G) * D}
        return {"bytes": T * D * (size + 2) * (H + G) + table, "flops": 8.0 * T * (H + G) * D}
    if c["kind"] == "self":
        # (lengths are even over a quarter of the longest to all of it, new tokens over a half to all)
        kept = c["longest"] * (1 + 0.625 * (c["B"] - 1))
        rows = c["B"] * c["new"] * (0.75 if c["new"] > 1 else 1.0)
        seen = kept / c["B"] - (0.375 * c["new"] if c["new"] > 1 else 0)
        return {"bytes": kept * G * D * 2 * 0.5625 + 4.0 * rows * H * D, "flops": 4.0 * rows * H * D * max(1.0, seen)}
    B, Tq, S = c["B"], c["Tq"], c["S"]
    part = {"none": 1.0, "lens": 0.75, "bytes": 0.8}[c["mask"]]
    return {"bytes": 4.0 * B * Tq * H * D + 4.0 * B * S * G * D * part, "flops": 4.0 * B * Tq * H * D * S * part}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def _exact_weights(packed, N, K, group):
    n, k = torch.arange(N, device="cuda")[:, None], torch.arange(K, device="cuda")[None]
    nt, kt = -(-N // 16), -(-K // 128)
    byte = ((n // 16 * kt + k // 128) * 64 + k % 32 // 8 * 16 + n % 16) * 16 + k % 128 // 32 * 4 + k % 2 * 2 + k % 8 // 4
    code = ((packed[byte].int() >> (k % 8 // 2 % 2 * 4)) & 15) - 8
    del byte
    s = packed[nt * kt * 1024:].view(torch.float16)[(n // 16 * (kt * 128 // group) + k // group) * 16 + n % 16]
    return code.double() * s.double()


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


def _exact_heads(q, k, v, visible):
    """q [rows, D], k, v [S, D], visible [rows or 1, S], of one head"""
    s = torch.where(visible, q @ k.t() / q.shape[1] ** 0.5, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
    w = torch.softmax(s, 1) @ v
    return torch.where(visible.any(1, keepdim=True), w, torch.zeros((), dtype=torch.float64, device="cuda"))


def exact(case, seed):
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "linear":
        rows = max(1, 2**25 // c["K"]) // 16 * 16 or 16
        kt, per, cut = -(-c["K"] // 128), 128 // c["group"], -(-c["N"] // 16) * -(-c["K"] // 128) * 1024
        ys = []
        for a in range(0, c["N"], rows):
            n = min(rows, c["N"] - a)
            t0, t1 = a // 16, -(-(a + n) // 16)
            part = torch.cat([st["packed"][t0 * kt * 1024:t1 * kt * 1024], st["packed"][cut:][t0 * kt * per * 32:t1 * kt * per * 32]])
            ys.append(st["X"].to(f64) @ _exact_weights(part, n, c["K"], c["group"]).t())
        y = torch.cat(ys, 1) + (0 if st["bias"] is None else st["bias"].to(f64))
        return y * torch.special.ndtr(y) if c["gelu"] else y
    H, G, D = c["heads"], c["kv_heads"], c["D"]
    if c["kind"] == "rope":
        x, R = st["qkv"].to(f64).view(c["T"], H + 2 * G, D), c["R"]
        y = x[:, :H + G].clone()
        if c["norm"]:
            y /= ((y**2).sum(-1, keepdim=True) / D + 1e-6).sqrt()
            y[:, :H] *= st["qw"].to(f64)
            y[:, H:] *= st["kw"].to(f64)
        at = st["positions"].long()
        turn = torch.complex(st["cos"].to(f64)[at], st["sin"].to(f64)[at])[:, None]
        i = torch.arange(R // 2, device="cuda")
        re, im = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + R // 2)
        z = torch.complex(y[..., re], y[..., im]) * turn
        y[..., re], y[..., im] = z.real, z.imag
        if not c["cache"]:
            return y[:, :H], y[:, H:]

        def held(x):
            out = torch.empty_like(x)
            for a in range(0, D, 32):
                part = x[..., a:a + 32]
                s = part.abs().amax(-1, keepdim=True) / 7
                m = torch.frexp(s).mantissa  # in 1/2 .. 1
                s = torch.round(m * 128) / 128 * (s / m)
                out[..., a:a + 32] = torch.round(part / s).clamp(-7, 7) * s
            return out

        return y[:, :H], held(y[:, H:]), held(x[:, H + G:])
    outs = []
    if c["kind"] == "self":
        cu, lens, table = st["cu_q"].tolist(), st["lens"].tolist(), st["block_table"].long()
        for b in range(c["B"]):
            n, L = cu[b + 1] - cu[b], lens[b]
            K, V = _exact_cache(st["cache"][table[b, :-(-L // _PAGE)]], D)  # [pages, G, 64, D]
            K, V = (x.transpose(0, 1).reshape(G, -1, D)[:, :L] for x in (K, V))
            seen = torch.arange(L, device="cuda")[None] <= L - n + torch.arange(n, device="cuda")[:, None]
            q = st["q"][cu[b]:cu[b + 1]].to(f64)
            outs.append(torch.stack([_exact_heads(q[:, h], K[h * G // H], V[h * G // H], seen) for h in range(H)], 1))
        return torch.cat(outs)
    for b in range(c["B"]):
        seen = torch.ones((1, c["S"]), dtype=torch.bool, device="cuda")
        if st["lens"] is not None:
            seen[:, int(st["lens"][b]):] = False
        if st["mask"] is not None:
            seen &= st["mask"][b:b + 1] != 0
        outs.append(torch.stack([_exact_heads(st["q"][b, :, h].to(f64), st["k"][b, :, h * G // H].to(f64), st["v"][b, :, h * G // H].to(f64), seen) for h in range(H)], 1))
    return torch.stack(outs)
