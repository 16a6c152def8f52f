"""Attention over the paged 4-bit cache and to an encoder's states, against the definition in 64 bits and what the kernels' own roundings allow."""
import numpy as np
import pytest

import decoder_reference as ref
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class _Cache:
    """A batch of sequences in pages of any order; places that no token has hold bytes of `fill` (0xFF: scales that are NaN)"""

    def __init__(self, lens, G, D, seed=0, sharp=1.0, fill=0xFF, spare=2):
        r = np.random.default_rng(seed + D)
        self.lens, self.G, self.D = lens, G, D
        per = max(1, max(-(-n // 64) for n in lens))
        total = sum(-(-n // 64) for n in lens) + spare
        order = iter(r.permutation(total))
        self.table = np.full((len(lens), per), 2**31 - 1, np.int32)  # entries that no token needs are no pages
        self.pages = np.full((total, G, 72 * ref.padded(D)), fill, np.uint8)
        self.K, self.V = [], []
        pl = ref.Places(D)
        for b, n in enumerate(lens):
            k = (r.standard_normal((n, G, D)) * sharp).astype(np.float32)
            v = (r.standard_normal((n, G, D)) + r.standard_normal((1, G, D))).astype(np.float32)
            (ck, sk), (cv, sv) = ref.cache_codes(k), ref.cache_codes(v)
            for i in range(-(-n // 64)):
                m = min(64, n - 64 * i)
                part = []
                for x in (ck, sk, cv, sv):
                    whole = np.zeros((1, G, 64, x.shape[-1]), x.dtype)
                    whole[0, :, :m] = x[64 * i:64 * i + m].transpose(1, 0, 2)
                    part.append(whole)
                new, page = ref.write_pages(*part, D)[0], next(order)
                self.table[b, i] = page
                for at in (pl.k_byte[:m], pl.v_byte[:m]):  # only what tokens hold (a byte of value codes is of one token)
                    self.pages[page][:, at] = new[:, at]
                for at in (pl.k_scale[:m], pl.v_scale[:m]):
                    self.pages[page].view(np.uint16)[:, at] = new.view(np.uint16)[:, at]
            s = lambda c, sc: c * sc.astype(np.float64).repeat(32, -1)[..., :D]  # noqa: E731
            self.K.append(s(ck, sk))
            self.V.append(s(cv, sv))

    def expected(self, q, counts, scale):
        """q [tokens, H, D]; counts: new tokens of each sequence"""
        out, off, at, H = np.zeros(q.shape), np.zeros(q.shape), 0, q.shape[1]
        for b, n in enumerate(counts):
            L = self.lens[b]
            seen = np.arange(L)[None] <= L - n + np.arange(n)[:, None]
            for h in range(H):
                out[at:at + n, h], off[at:at + n, h] = ref.attend(q[at:at + n, h].astype(np.float64), self.K[b][:, h * self.G // H], self.V[b][:, h * self.G // H], seen, scale)
            at += n
        return out, off


def _run(g, c, q, counts, scale=None, cu=True, **kw):
    cu_q = dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)) if cu else None
    return g.attention_kv4(dev(q), dev(c.pages), dev(c.table), dev(np.array(c.lens, np.int32)), cu_q=cu_q, max_q=max(max(counts), 1), scale=scale, **kw)


def _check(y, exp, off):
    y = host(y).astype(np.float64)
    assert (np.abs(y - exp) <= off).all(), np.max(np.abs(y - exp) / off)


# heads that share a key head: one, some, an odd number, more than a block of 16; heads of every padding
HEADS = [(4, 4, 64), (8, 2, 128), (6, 2, 80), (7, 1, 256), (20, 1, 128), (3, 1, 40), (2, 2, 136)]


@pytest.mark.parametrize("H,G,D", HEADS)
def test_one_token_a_sequence(g, H, G, D):
    """Lengths at the edges of tiles (32) and pages (64), none and one among them"""
    lens = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 300]
    c = _Cache(lens, G, D)
    q = np.random.default_rng(H).standard_normal((len(lens), H, D)).astype(np.float16)
    exp, off = c.expected(q, [1] * len(lens), D ** -0.5)
    for cu in (False, True):
        y = _run(g, c, q, [1] * len(lens), cu=cu)
        _check(y, exp, off)
        assert not host(y)[0].any()


@pytest.mark.parametrize("H,G,D", HEADS)
def test_several_tokens_a_sequence(g, H, G, D):
    """Ragged new tokens: none, one, a chunk that is the whole history, more queries than the history has, chunks across pages"""
    lens, counts = [40, 7, 5, 130, 3, 200, 64], [0, 1, 5, 35, 6, 70, 64]
    c = _Cache(lens, G, D, seed=1)
    q = np.random.default_rng(H + 1).standard_normal((sum(counts), H, D)).astype(np.float16)
    _check(_run(g, c, q, counts), *c.expected(q, counts, D ** -0.5))


@pytest.mark.parametrize("batch,longest,H,G,D", [(1, 5000, 8, 2, 64), (2, 9001, 4, 1, 128), (1, 20001, 4, 2, 80), (3, 2500, 2, 1, 256)])
def test_long_histories_are_cut_and_joined(g, batch, longest, H, G, D):
    lens = [longest, 70, 1024][:batch]
    assert g.lib().gpusq_attention_kv4_workspace_bytes(batch, batch, 1, -(-longest // 64), H, G, D) > 0
    c = _Cache(lens, G, D, seed=2)
    q = np.random.default_rng(9).standard_normal((batch, H, D)).astype(np.float16)
    exp, off = c.expected(q, [1] * batch, D ** -0.5)
    y = _run(g, c, q, [1] * batch)
    _check(y, exp, off)
    ws = torch.full((g.lib().gpusq_attention_kv4_workspace_bytes(batch, batch, 1, c.table.shape[1], H, G, D),), 255, dtype=torch.uint8, device="cuda")  # NaN
    out = torch.full((batch, H, D), 7, dtype=torch.float16, device="cuda")
    assert torch.equal(_run(g, c, q, [1] * batch, workspace=ws, out=out), y)
    counts = [5, 3, 17][:batch]
    q = np.random.default_rng(10).standard_normal((sum(counts), H, D)).astype(np.float16)
    _check(_run(g, c, q, counts), *c.expected(q, counts, D ** -0.5))


@pytest.mark.parametrize("sharp", [0.0, 8.0, 60.0])
def test_flat_and_sharp_scores(g, sharp):
    """All scores alike; scores hundreds apart, whose maximum moves from tile to tile"""
    lens = [700, 33]
    c = _Cache(lens, 2, 128, seed=3, sharp=sharp)
    q = (np.random.default_rng(11).standard_normal((2, 8, 128)) * 2).astype(np.float16)
    for scale in (None, 0.5, 1e-4):
        _check(_run(g, c, q, [1, 1], scale=scale), *c.expected(q, [1, 1], 128 ** -0.5 if scale is None else scale))


def test_a_rising_maximum(g):
    """Keys that grow along the history: every tile has a new maximum"""
    G, D, n = 1, 64, 640
    c = _Cache([n], G, D, seed=4)
    k = (np.linspace(0.1, 6, n)[:, None, None] * np.ones((n, 1, D))).astype(np.float32)
    v = np.random.default_rng(1).standard_normal((n, 1, D)).astype(np.float32)
    (ck, sk), (cv, sv) = ref.cache_codes(k), ref.cache_codes(v)
    pages = [x.reshape(n // 64, 64, 1, -1).transpose(0, 2, 1, 3) for x in (ck, sk, cv, sv)]
    c.pages, c.table = ref.write_pages(*pages, D), np.arange(n // 64, dtype=np.int32)[None]
    s = lambda x, sc: x * sc.astype(np.float64).repeat(32, -1)  # noqa: E731
    c.K, c.V = [s(ck, sk)], [s(cv, sv)]
    for sign in (1, -1):
        q = np.full((3, 2, D), sign, np.float16)
        _check(_run(g, c, q, [3]), *c.expected(q, [3], D ** -0.5))


def test_pages_that_are_none(g):
    """Table entries outside the cache: their tokens are not seen, and nothing is read there"""
    c = _Cache([200, 90], 1, 64, seed=5)
    q = np.random.default_rng(12).standard_normal((2, 4, 64)).astype(np.float16)
    c.table[0, 1], c.table[1, 0], c.table[1, 1] = -1, 10**9, len(c.pages)
    hidden = slice(64, 128)
    c.K[0][hidden], c.V[0][hidden] = 0, 0
    y = host(_run(g, c, q, [1, 1]))
    seen = np.ones((1, 200), bool)
    seen[:, hidden] = False
    for h in range(4):
        exp, off = ref.attend(q[0:1, h].astype(np.float64), c.K[0][:, 0], c.V[0][:, 0], seen, 64 ** -0.5)
        assert (np.abs(y[0:1, h] - exp) <= off).all()
    assert not y[1].any()


def test_lengths_and_offsets_out_of_range_stay_inside(g):
    """A length beyond the table is cut to it, a negative one is 0; queries that no token of q has are not answered, nor those beyond max_q"""
    c = _Cache([64, 64, 64], 1, 64, seed=6)
    q = np.random.default_rng(13).standard_normal((4, 2, 64)).astype(np.float16)
    lens = dev(np.array([2**31 - 1, -7, 64], np.int32))
    out = torch.full((4, 2, 64), 7, dtype=torch.float16, device="cuda")
    cu = dev(np.array([0, 1, 2, 4], np.int32))
    y = host(g.attention_kv4(dev(q), dev(c.pages), dev(c.table), lens, cu_q=cu, max_q=1, out=out))
    exp, off = c.expected(q[:1], [1], 64 ** -0.5)
    assert (np.abs(y[:1] - exp) <= off).all() and not y[1].any() and (y[3] == 7).all()
    for cu in ([-1, 1, 2, 3], [0, 5, 9, 2**31 - 1], [3, 2, 1, 0]):
        y = host(g.attention_kv4(dev(q), dev(c.pages), dev(c.table), lens, cu_q=dev(np.array(cu, np.int32)), max_q=2))
        assert y.shape == (4, 2, 64)


def test_offsets_beyond_32_bits(g):
    """Pages and queries more than 4 GiB into their tensors"""
    D, G = 128, 8
    per_page = G * 72 * D
    pages = 2**32 // per_page + 70
    cache = torch.full((pages, G, 72 * D), 255, dtype=torch.uint8, device="cuda")
    c = _Cache([100], G, D, seed=7)
    last = pages - len(c.pages)
    cache[last:] = dev(c.pages)
    c.table = np.where(c.table < len(c.pages), c.table + last, c.table).astype(np.int32)
    q = np.random.default_rng(14).standard_normal((1, 8, D)).astype(np.float16)
    exp, off = c.expected(q, [1], D ** -0.5)
    _check(g.attention_kv4(dev(q), cache, dev(c.table), dev(np.array([100], np.int32))), exp, off)
    # and a token appended there
    x = np.random.default_rng(15).standard_normal((1, 3 * G * D)).astype(np.float16)
    slot = pages * 64 - 5
    _, k, v = g.qk_norm_rope(dev(x), G, G, D, cache=cache, slots=dev(np.array([slot], np.int32)), want_cached=True)
    K, V = ref.read_pages(host(cache[-1:]), D)
    assert np.array_equal(host(k)[0].astype(np.float64), K[0, :, 59]) and np.array_equal(host(v)[0].astype(np.float64), V[0, :, 59])


# ---- to an encoder's states ------------------------------------------------------------------------------------------------------------


def _cross_expected(q, k, v, seen, scale):
    out, off = np.zeros(q.shape), np.zeros(q.shape)
    H, G = q.shape[2], k.shape[2]
    for b in range(q.shape[0]):
        for h in range(H):
            s = np.broadcast_to(seen[b][None], (q.shape[1], k.shape[1]))
            out[b, :, h], off[b, :, h] = ref.attend(q[b, :, h].astype(np.float64), k[b, :, h * G // H].astype(np.float64), v[b, :, h * G // H].astype(np.float64), s, scale)
    return out, off


def _normal(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape).astype(np.float16)


# one query, some, blocks that are not full; keys at the edges of a tile; one key head for many and for one
@pytest.mark.parametrize("B,Tq,S,H,G,D", [(1, 1, 1, 1, 1, 64), (2, 1, 257, 16, 16, 80), (3, 5, 31, 4, 2, 64), (1, 16, 33, 2, 2, 128), (2, 17, 64, 6, 2, 96), (1, 70, 65, 3, 1, 128),
                                           (2, 197, 197, 3, 3, 64), (1, 130, 300, 4, 1, 256), (1, 33, 95, 7, 1, 40), (1, 200, 129, 2, 1, 72), (5, 3, 100, 34, 2, 64)])
@pytest.mark.parametrize("mask", ["none", "lens", "bytes", "both"])
def test_cross(g, B, Tq, S, H, G, D, mask):
    q, k, v = _normal(B, B, Tq, H, D), _normal(S, B, S, G, D), _normal(D, B, S, G, D)
    r = np.random.default_rng(S + D)
    seen = np.ones((B, S), bool)
    lens = bytes_ = None
    if mask in ("lens", "both"):
        lens = r.integers(0, S + 1, B).astype(np.int32)
        lens[-1] = 0 if B > 1 else S
        seen &= np.arange(S)[None] < lens[:, None]
    if mask in ("bytes", "both"):
        bytes_ = (r.random((B, S)) < 0.6).astype(np.uint8) * 3
        bytes_[0] = 0 if B > 2 else bytes_[0]
        seen &= bytes_ != 0
    k[~seen], v[~seen] = np.nan, np.inf  # what is not seen may hold anything
    y = g.cross_attention(dev(q), dev(k), dev(v), kv_lens=None if lens is None else dev(lens), key_mask=None if bytes_ is None else dev(bytes_))
    exp, off = _cross_expected(q, np.where(seen[..., None, None], k, 0), np.where(seen[..., None, None], v, 0), seen, D ** -0.5)
    _check(y, exp, off)
    assert not host(y)[~seen.any(1)].any()
    if bytes_ is not None and lens is None:
        assert torch.equal(y, g.cross_attention(dev(q), dev(k), dev(v), key_mask=dev(bytes_ != 0)))


@pytest.mark.parametrize("Tq,S,D", [(1, 40, 64), (50, 70, 64), (20, 33, 128)])
def test_strides(g, Tq, S, D):
    """Heads in a packed projection, heads apart from each other, batches shared, keys repeated by a stride of 0"""
    B, H = 2, 4
    q, k, v = _normal(1, B, Tq, H, D), _normal(2, B, S, H, D), _normal(3, B, S, H, D)
    exp, off = _cross_expected(q, k, v, np.ones((B, S), bool), D ** -0.5)
    packed = torch.cat([dev(k), dev(v)], 2)
    apart = dev(q).transpose(1, 2).contiguous().transpose(1, 2)
    for a, b, c in ((dev(q), packed[:, :, :H], packed[:, :, H:]), (apart, dev(k).transpose(1, 2).contiguous().transpose(1, 2), dev(v))):
        _check(g.cross_attention(a, b, c), exp, off)
    one = g.cross_attention(dev(q), dev(k[:1]).expand(B, S, H, D), dev(v[:1]).expand(B, S, H, D))
    exp, off = _cross_expected(q, np.repeat(k[:1], B, 0), np.repeat(v[:1], B, 0), np.ones((B, S), bool), D ** -0.5)
    _check(one, exp, off)
    wide = torch.zeros((B, S, H, 3 * D + 8), dtype=torch.float16, device="cuda")
    wide[..., 8:8 + D] = dev(k)
    _check(g.cross_attention(dev(q), wide[..., 8:8 + D], dev(v), scale=0.3), *_cross_expected(q, k, v, np.ones((B, S), bool), 0.3))


def test_long_states_are_cut_and_joined(g):
    B, Tq, S, H, G, D = 1, 2, 6001, 4, 2, 64
    assert g.lib().gpusq_cross_attention_workspace_bytes(B, Tq, S, H, G, D) > 0
    q, k, v = _normal(4, B, Tq, H, D), _normal(5, B, S, G, D), _normal(6, B, S, G, D)
    for lens in (None, [4100], [1], [0]):
        seen = np.arange(S)[None] < (S if lens is None else lens[0])
        y = g.cross_attention(dev(q), dev(k), dev(v), kv_lens=None if lens is None else dev(np.array(lens, np.int32)))
        _check(y, *_cross_expected(q, k, v, seen, D ** -0.5))


# many columns of every padding, histories and states cut into parts; what no key leaves anything for, a whole part among it
@pytest.mark.parametrize("D", [64, 128, 200])
def test_many_queries_over_parts(g, D):
    counts, lens, H, G = [90, 40], [2100, 90], 4, 1
    assert g.lib().gpusq_attention_kv4_workspace_bytes(sum(counts), 2, 90, -(-2100 // 64), H, G, D) > 0
    c = _Cache(lens, G, D, seed=31)
    q = np.random.default_rng(32).standard_normal((sum(counts), H, D)).astype(np.float16)
    _check(_run(g, c, q, counts), *c.expected(q, counts, D ** -0.5))
    B, Tq, S = 2, 45, 1500
    assert g.lib().gpusq_cross_attention_workspace_bytes(B, Tq, S, H, G, D) > 0
    q, k, v = _normal(33, B, Tq, H, D), _normal(34, B, S, G, D), _normal(35, B, S, G, D)
    bytes_ = (np.random.default_rng(36).random((B, S)) < 0.5).astype(np.uint8)
    bytes_[0, :700], bytes_[1, 400:] = 0, 0
    lens = np.array([1203, 1500], np.int32)
    for use_lens, use_bytes in ((False, False), (True, False), (False, True), (True, True)):
        seen = np.ones((B, S), bool)
        if use_lens:
            seen &= np.arange(S)[None] < lens[:, None]
        if use_bytes:
            seen &= bytes_ != 0
        a, b = (np.where(seen[..., None, None], x, np.float16(np.nan)) for x in (k, v))
        y = g.cross_attention(dev(q), dev(a), dev(b), kv_lens=dev(lens) if use_lens else None, key_mask=dev(bytes_) if use_bytes else None)
        _check(y, *_cross_expected(q, np.where(seen[..., None, None], k, 0), np.where(seen[..., None, None], v, 0), seen, D ** -0.5))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Tq", [10, 90])
def test_masks_that_hide_whole_tiles(g, D, Tq):
    """Keys seen only at the end, at the beginning, one here and there, none: hidden ones hold NaN"""
    B, S, H = 4, 230, 2
    seen = np.zeros((B, S), bool)
    seen[0, 200:], seen[1, :3], seen[2, [0, 63, 64, 129, 229]] = True, True, True
    q, k, v = _normal(41, B, Tq, H, D), _normal(42, B, S, 1, D), _normal(43, B, S, 1, D)
    y = g.cross_attention(dev(q), *(dev(np.where(seen[..., None, None], x, np.float16(np.nan))) for x in (k, v)), key_mask=dev(seen))
    _check(y, *_cross_expected(q, k, v, seen, D ** -0.5))
    assert not host(y)[3].any()


def test_states_far_apart(g):
    """A stride of 2^24 values from token to token, for few queries and many"""
    S, D = 40, 64
    big = torch.zeros(S * 2**24, dtype=torch.float16, device="cuda")
    far = big.as_strided((1, S, 1, D), (0, 2**24, D, 1))
    k, v = _normal(51, 1, S, 1, D), _normal(52, 1, S, 1, D)
    far.copy_(dev(k))
    for Tq in (3, 50):
        q = _normal(53, 1, Tq, 2, D)
        exp, off = _cross_expected(q, k, v, np.ones((1, S), bool), D ** -0.5)
        _check(g.cross_attention(dev(q), far, dev(v)), exp, off)
        exp, off = _cross_expected(q, v, k, np.ones((1, S), bool), D ** -0.5)
        _check(g.cross_attention(dev(q), dev(v), far), exp, off)


def test_infinite_and_nan_operands_keep_to_their_rows(g):
    q, k, v = _normal(7, 1, 40, 2, 64), _normal(8, 1, 70, 2, 64), _normal(9, 1, 70, 2, 64)
    clean = host(g.cross_attention(dev(q), dev(k), dev(v)))
    q[0, 3, 0, 5], q[0, 20, 1, 1] = np.nan, np.inf
    y = host(g.cross_attention(dev(q), dev(k), dev(v)))
    assert np.isnan(y[0, 3, 0]).all() and np.array_equal(y[0, 3, 1], clean[0, 3, 1])
    rest = [i for i in range(40) if i not in (3, 20)]
    assert np.array_equal(y[0, rest], clean[0, rest])


def test_on_another_stream_and_in_a_graph(g):
    """The calls on a stream of their own, and replayed from a graph on new inputs between eager work, each replay like the eager call"""
    q, k, v = (dev(_normal(s, *shape)) for s, shape in ((1, (2, 1, 8, 64)), (2, (2, 4000, 2, 64)), (3, (2, 4000, 2, 64))))
    c = _Cache([3000, 77], 2, 64, seed=8)
    pages, table, lens = dev(c.pages), dev(c.table), dev(np.array(c.lens, np.int32))
    run = lambda: (g.cross_attention(q, k, v), g.attention_kv4(q[:, 0], pages, table, lens))  # noqa: E731
    eager = run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for i in range(4):
        q.copy_(dev(_normal(20 + i, 2, 1, 8, 64)))
        lens.copy_(dev(np.array([3000 - 700 * i, 77], np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        got = [h.clone() for h in held]
        assert all(torch.equal(a, b) for a, b in zip(got, run()))
        torch.cuda.synchronize()


def test_refusals(g):
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = g.kv4_cache(4, 2, 64)
    ok = dict(q=f16(2, 4, 64), cache=cache, block_table=i32(2, 2), kv_lens=i32(2))
    assert g.attention_kv4(**ok).shape == (2, 4, 64)
    for change in (dict(q=f16(2, 4, 128)), dict(q=f16(2, 4, 64).float()), dict(cache=cache[:, :, :-16]), dict(block_table=i32(2, 2).long()), dict(kv_lens=i32(3)),
                   dict(cu_q=i32(2)), dict(block_table=i32(2, 4)[:, ::2]), dict(out=f16(2, 4, 32)), dict(q=f16(2, 4, 64).cpu()), dict(kv_lens=i32(2).cpu())):
        with pytest.raises(ValueError):
            g.attention_kv4(**{**ok, **change})
    for change in (dict(q=f16(2, 3, 64)), dict(q=f16(3, 4, 64)), dict(max_q=3), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(g.GpusqError):
            g.attention_kv4(**{**ok, **change})
    ok = dict(q=f16(2, 3, 4, 64), k=f16(2, 5, 2, 64), v=f16(2, 5, 2, 64))
    assert g.cross_attention(**ok).shape == (2, 3, 4, 64)
    for change in (dict(k=f16(2, 5, 2, 32)), dict(v=f16(2, 6, 2, 64)), dict(k=f16(1, 5, 2, 64), v=f16(1, 5, 2, 64)), dict(q=f16(2, 3, 4, 64).float()), dict(kv_lens=i32(3)),
                   dict(key_mask=i32(2, 5)), dict(key_mask=torch.zeros((2, 4), dtype=torch.uint8, device="cuda")), dict(q=f16(2, 3, 64, 4).transpose(2, 3)), dict(k=f16(2, 5, 2, 64).cpu())):
        with pytest.raises(ValueError):
            g.cross_attention(**{**ok, **change})
    for change in (dict(q=f16(2, 3, 3, 64)), dict(scale=-0.5), dict(q=f16(2, 3, 4, 68)[..., :64])):
        with pytest.raises(g.GpusqError):
            g.cross_attention(**{**ok, **change})
    with pytest.raises(g.GpusqError):
        g.cross_attention(f16(1, 1, 1, 264), f16(1, 1, 1, 264), f16(1, 1, 1, 264))


def _repeated(table, batch):
    return dev(np.repeat(table, batch, 0))


# how many sequences leave room for so many parts (few queries, many queries to states, many over the cache)
PARTS = {1: (256, 300, 200), 2: (128, 200, 100), 8: (32, 64, 32), 9: (29, 56, 28)}


@pytest.mark.parametrize("parts", sorted(PARTS))
@pytest.mark.parametrize("Tq", [1, 40])
def test_a_query_that_is_no_number_stays_one_over_parts(g, parts, Tq):
    """Keys in one piece, in few parts and in many: a query with a NaN has no answer in any, and the others have theirs; keys that are no
    numbers in one part only leave no query an answer"""
    S, D = 4608, 64
    B = PARTS[parts][0 if Tq == 1 else 1]
    assert g.lib().gpusq_cross_attention_workspace_bytes(B, Tq, S, 1, 1, D) == (parts > 1) * parts * B * Tq * (D + 2) * 4
    q, k, v = _normal(61, B, Tq, 1, D), _normal(62, 1, S, 1, D), _normal(63, 1, S, 1, D)
    whole = lambda x: dev(x).expand(B, S, 1, D)  # noqa: E731
    clean = host(g.cross_attention(dev(q), whole(k), whole(v)))
    broken = q.copy()
    broken[1, 0, 0, 5] = np.nan
    y = host(g.cross_attention(dev(broken), whole(k), whole(v)))
    assert np.isnan(y[1, 0]).all()
    assert np.array_equal(np.delete(y, 1, 0), np.delete(clean, 1, 0))
    exp, off = _cross_expected(q[1:2, 1:], k, v, np.ones((1, S), bool), D ** -0.5)
    assert (np.abs(y[1:2, 1:] - exp) <= off).all()
    k[:, -(S // parts):] = np.nan
    assert np.isnan(host(g.cross_attention(dev(q), whole(k), whole(v)))).all()

    B = PARTS[parts][0 if Tq == 1 else 2]
    assert g.lib().gpusq_attention_kv4_workspace_bytes(B * Tq, B, Tq, S // 64, 1, 1, D) == (parts > 1) * parts * B * Tq * (D + 2) * 4
    c = _Cache([S], 1, D, seed=64)
    args = dev(c.pages), _repeated(c.table, B), dev(np.full(B, S, np.int32))
    q = _normal(65, B * Tq, 1, D)
    clean = host(g.attention_kv4(dev(q), *args, max_q=Tq))
    broken = q.copy()
    broken[Tq, 0, 5] = np.nan
    y = host(g.attention_kv4(dev(broken), *args, max_q=Tq))
    assert np.isnan(y[Tq]).all()
    rest = np.delete(np.arange(B * Tq), np.arange(Tq, 2 * Tq))
    assert np.array_equal(y[rest], clean[rest])
    exp, off = c.expected(q[Tq:2 * Tq], [Tq], D ** -0.5)
    assert (np.abs(y[Tq + 1:2 * Tq] - exp[1:]) <= off[1:]).all()


def test_columns_whose_products_pass_32_bits(g):
    """Three million columns of one key head: every row is answered, from its own query"""
    n, H, D, S = 47000, 64, 64, 40
    c = _Cache([S], 1, D, seed=66)
    q = torch.randn((n, H, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    out = torch.full((n, H, D), 7, dtype=torch.float16, device="cuda")
    g.attention_kv4(q, dev(c.pages), dev(c.table), dev(np.array([S], np.int32)), max_q=n, out=out)
    exp, off = c.expected(host(q[-S:]), [S], D ** -0.5)  # the last queries see the tokens, those before them nothing
    _check(out[-S:], exp, off)
    assert not out[:-S].any()
    k, v = _normal(67, 1, S, 1, D), _normal(68, 1, S, 1, D)
    out.fill_(7)
    g.cross_attention(q[None], dev(k), dev(v), out=out[None])
    K, V = dev(k)[0, :, 0].double(), dev(v)[0, :, 0].double()
    for a in range(0, n, 4700):  # the bounds of decoder_reference.attend
        x = q[a:a + 4700].double().view(-1, D)
        w = torch.softmax(x @ K.t().contiguous() * D ** -0.5, 1)
        delta = 2 * D * 2.0 ** -24 * D ** -0.5 * (x.abs() @ K.abs().t().contiguous())
        y = w @ V
        off = (w * (2.0 ** -11 + 2.0 ** -20 + delta + (w * delta).sum(1, keepdim=True))) @ V.abs() + 2.0 ** -31 * V.abs().sum(0) + 2.0 ** -11 * y.abs() + 2.0 ** -24
        assert ((out[a:a + 4700].double().view(-1, D) - y).abs() <= off).all()


# of few queries and many, over keys in one piece and in parts
@pytest.mark.parametrize("lens,counts,max_q", [([300, 64, 9], [5, 2, 1], 1), ([300, 64, 7], [5, 2, 7], 3), ([9001, 70], [6, 2], 2), ([400, 130], [70, 41], 40), ([5000, 90], [120, 33], 50)])
def test_more_new_tokens_than_max_q(g, lens, counts, max_q):
    """The first max_q of a sequence are answered, as what they are: they do not see the tokens behind them.  Without max_q all are."""
    G, D, H = 1, 64, 2
    c = _Cache(lens, G, D, seed=71)
    q = _normal(72, sum(counts), H, D)
    exp, off = c.expected(q, counts, D ** -0.5)
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    args = dev(q), dev(c.pages), dev(c.table), dev(np.array(lens, np.int32)), dev(cu)
    y = host(g.attention_kv4(*args, max_q=max_q)).astype(np.float64)
    answered = np.concatenate([np.arange(a, min(a + max_q, b)) for a, b in zip(cu, cu[1:])])
    assert (np.abs(y[answered] - exp[answered]) <= off[answered]).all()  # (the others hold anything)
    y = host(g.attention_kv4(*args)).astype(np.float64)
    assert (np.abs(y - exp) <= off).all()


def test_strides_of_dimensions_of_one(g):
    """What such a dimension has as its stride is never used, and may be anything"""
    S, D = 70, 64
    q, k, v = _normal(81, 1, 1, 1, D), _normal(82, 1, S, 1, D), _normal(83, 1, S, 1, D)
    odd = lambda x: dev(x).as_strided(x.shape, tuple(3 if n == 1 else s for n, s in zip(x.shape, dev(x).stride())))  # noqa: E731
    assert odd(k).stride() == (3, D, 3, 1)
    assert torch.equal(g.cross_attention(odd(q), odd(k), odd(v)), g.cross_attention(dev(q), dev(k), dev(v)))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Tq,S", [(3, 100), (50, 100), (50, 1500)])
def test_a_query_that_sees_nothing_and_is_no_number(g, Tq, S, D):
    """0, as for any query that sees nothing, where a mask or a length hides all keys, which hold anything, one piece or parts"""
    B = 3
    q, k, v = _normal(91, B, Tq, 2, D), _normal(92, B, S, 1, D), _normal(93, B, S, 1, D)
    seen = np.ones((B, S), bool)
    seen[1] = False
    q[:, 1, 0, 3], q[:, 2, 1, 4], k[1], v[1] = np.nan, np.inf, np.nan, np.nan
    for hide in (dict(key_mask=dev(seen)), dict(kv_lens=dev(np.array([S, 0, S], np.int32))), dict(key_mask=dev(seen), kv_lens=dev(np.array([S, 5, S], np.int32)))):
        y = host(g.cross_attention(dev(q), dev(k), dev(v), **hide))
        assert not y[1].any()
        assert np.isnan(y[[0, 2], 1, 0]).all() and np.isfinite(y[[0, 2], 0]).all()


# scores up to millions, of either sign; one piece and parts, few queries and many
@pytest.mark.parametrize("size", [30.0, 300.0])
@pytest.mark.parametrize("Tq,S,D", [(3, 70, 64), (40, 70, 128), (40, 1600, 64), (2, 3000, 256), (1, 9000, 64)])
def test_large_scores(g, Tq, S, D, size):
    """Keys that are multiples of one vector, so that the scores of a query are as far apart as the multiples: the largest takes all (the next one is
    32-bit roundings of a sum away many times over)"""
    r = np.random.default_rng(D + S)
    u = np.where(r.random(D) < 0.5, 1.0, 0.5)
    some = np.sort(r.choice(S, min(S, 60), replace=False))
    a = np.full(S, -1.0)
    a[some] = r.permutation(np.linspace(0.25, 1, len(some)))  # (the others: far below or, for queries of the other sign, far above in one place)
    a[some[0] if some[0] != S - 1 else 0] = -2.0
    k = (np.float16(size) * a[:, None] * u)[None, :, None].astype(np.float16)
    sign = np.where(np.arange(Tq) % 2 == 0, 1.0, -1.0)
    q = (size * sign[:, None] * np.ones(D))[None, :, None].astype(np.float16)
    v = r.standard_normal((1, S, 1, D)).astype(np.float16)
    scores = (q[0, :, 0].astype(np.float64) @ k[0, :, 0].astype(np.float64).T) * D ** -0.5
    order = np.sort(scores, 1)
    exp, off = _cross_expected(q, k, v, np.ones((1, S), bool), D ** -0.5)
    near = (order[:, -1] - order[:, -2]) > np.maximum(40, 4 * D * 2.0 ** -24 * np.abs(order).max(1))
    assert size < 300 or near.all()
    y = host(g.cross_attention(dev(q), dev(k), dev(v))).astype(np.float64)
    assert np.isfinite(y).all()
    best = v[0, scores.argmax(1), 0].astype(np.float64)
    assert (np.abs(y[0, near, 0] - best[near]) <= 2.0 ** -10 * np.abs(best[near]) + 2.0 ** -24).all()
    assert (np.abs(y - exp) <= off)[:, ~near].all()


@pytest.mark.parametrize("Tq,S", [(1, 200), (40, 200), (1, 9000), (40, 2100)])
def test_large_scores_over_the_cache(g, Tq, S):
    """The same where the keys are the cache's largest, 7 times 896"""
    D = 64
    c = _Cache([S], 1, D, seed=95)
    best = S // 3
    k = np.full((S, 1, D), -896.0 * 7, np.float32)
    k[best] = 896.0 * 7  # seen by the last queries; the ones in front of it have only keys that are alike
    (ck, sk), (cv, sv) = ref.cache_codes(k), ref.cache_codes(np.random.default_rng(3).standard_normal((S, 1, D)).astype(np.float32))
    n = -(-S // 64)
    pages = [np.concatenate([x, np.zeros((n * 64 - S,) + x.shape[1:], x.dtype)]).reshape(n, 64, 1, -1).transpose(0, 2, 1, 3) for x in (ck, sk, cv, sv)]
    c.pages, c.table = ref.write_pages(*pages, D), np.arange(n, dtype=np.int32)[None]
    V = cv * sv.astype(np.float64).repeat(32, -1)
    q = np.full((Tq, 1, D), 64.0, np.float16)  # scores of 3.2 million
    y = host(g.attention_kv4(dev(q), dev(c.pages), dev(c.table), dev(np.array([S], np.int32)), max_q=Tq)).astype(np.float64)
    assert (np.abs(y[:, 0] - V[best, 0]) <= 2.0 ** -10 * np.abs(V[best, 0]) + 2.0 ** -24).all()
    y = host(g.attention_kv4(dev(-q), dev(c.pages), dev(c.table), dev(np.array([S], np.int32)), max_q=Tq)).astype(np.float64)
    for i in range(Tq):  # all but one alike: their mean, the weights' roundings at most 2^-11 of each
        seen = np.delete(np.arange(S - Tq + 1 + i), best)
        assert (np.abs(y[i, 0] - V[seen, 0].mean(0)) <= 2.0 ** -10 * np.abs(V[seen, 0]).mean(0) + 2.0 ** -24).all()
