"""Norms of queries and keys per head, rotation, and the append to the 4-bit cache, against their definition in 64 bits."""
import numpy as np
import pytest

import decoder_reference as ref
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class _Case:
    def __init__(self, T, H, G, D, R, dtype=np.float16, norm=True, weights=True, table=50, seed=0):
        r = np.random.default_rng(seed + T + D)
        self.T, self.H, self.G, self.D, self.R, self.norm = T, H, G, D, R, norm
        self.x = (r.standard_normal((T, (H + 2 * G) * D)) * 1.5).astype(dtype)
        self.qw, self.kw = [(1 + 0.2 * r.standard_normal(D)).astype(np.float32) for _ in range(2)] if weights else (None, None)
        a = r.uniform(0, 6.3, (table, R // 2))
        self.cos, self.sin = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
        self.pos = r.integers(0, table, T).astype(np.int32)
        self.eps = 1e-5

    def kwargs(self, interleaved):
        kw = dict(norm=self.norm, eps=self.eps, interleaved=interleaved)
        if self.qw is not None:
            kw.update(q_weight=dev(self.qw), k_weight=dev(self.kw))
        if self.R:
            kw.update(cos=dev(self.cos), sin=dev(self.sin), positions=dev(self.pos))
        return kw

    def expected(self, interleaved):
        T, H, G, D = self.T, self.H, self.G, self.D
        x = self.x.reshape(T, H + 2 * G, D)
        c, s = self.cos[self.pos], self.sin[self.pos]
        how = (self.eps, c, s, self.R, interleaved)
        return ref.norm_rope(x[:, :H], self.norm, self.qw, *how), ref.norm_rope(x[:, H:H + G], self.norm, self.kw, *how), x[:, H + G:]


def _near(y, exp, D):
    """One rounding to fp16; a pair's turn adds two products, each off by a few 2^-24 of itself (norm: the sum of D squares, half of it)"""
    size = np.sqrt((exp ** 2).max()) * 2
    off = 2.0 ** -11 * np.abs(exp) + 2.0 ** -25 + (D / 2 + 8) * 2.0 ** -24 * size
    return (np.abs(y.astype(np.float64) - exp) <= off).all()


SIZES = [(1, 4, 4, 64, 64), (3, 8, 2, 128, 128), (65, 6, 3, 80, 80), (7, 4, 1, 96, 48), (5, 2, 2, 256, 128), (2, 3, 3, 8, 8), (9, 5, 1, 40, 0), (33, 16, 16, 136, 136), (300, 2, 1, 72, 24)]


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,G,D,R", SIZES)
def test_without_a_cache(g, T, H, G, D, R, interleaved, dtype):
    for norm, weights in ((True, True), (True, False), (False, False)):
        c = _Case(T, H, G, D, R, dtype, norm, weights)
        q, k = g.qk_norm_rope(dev(c.x), H, G, D, **c.kwargs(interleaved))
        eq, ek, _ = c.expected(interleaved)
        assert _near(host(q), eq, D) and _near(host(k), ek, D)


def test_rows_of_a_wider_tensor(g):
    c = _Case(11, 4, 2, 64, 64)
    wide = np.full((11, 8 * 64 + 72), 9, np.float16)
    wide[:, 8:8 + 8 * 64] = c.x
    q, k = g.qk_norm_rope(dev(wide)[:, 8:8 + 8 * 64], 4, 2, 64, **c.kwargs(False))
    q0, k0 = g.qk_norm_rope(dev(c.x), 4, 2, 64, **c.kwargs(False))
    assert torch.equal(q, q0) and torch.equal(k, k0)


def _slots(T, pages, seed):
    return np.random.default_rng(seed).permutation(pages * 64)[:T].astype(np.int32)


def _gather(pages, slots, D):
    """K, V [T, heads, D] of the slots, and their scales"""
    K, V = ref.read_pages(pages, D)
    p = ref.Places(D)
    halves = pages.view(np.float16)
    at = lambda x: x[slots // 64, :, slots % 64]  # noqa: E731
    return at(K), at(V), at(halves[..., p.k_scale]), at(halves[..., p.v_scale])


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,G,D,R", SIZES)
def test_into_the_cache(g, T, H, G, D, R, interleaved, dtype):
    for norm in (True, False):
        c = _Case(T, H, G, D, R, dtype, norm)
        pages = -(-T // 64) + 2
        cache = g.kv4_cache(pages, G, D)
        cache.fill_(0x5A)
        slots = _slots(T, pages, D)
        q, k, v = g.qk_norm_rope(dev(c.x), H, G, D, **c.kwargs(interleaved), cache=cache, slots=dev(slots), want_cached=True)
        eq, ek, ev = c.expected(interleaved)
        assert _near(host(q), eq, D)
        K, V, ks, vs = _gather(host(cache), slots, D)
        # what comes back is what the cache stands for, exactly, channels beyond the head are zeros
        assert np.array_equal(host(k).astype(np.float64), K) and np.array_equal(host(v).astype(np.float64), V)
        full = ref.read_pages(host(cache), ref.padded(D))
        assert not any(x[slots // 64, :, slots % 64, D:].any() for x in full)
        # values are quantised as they are: the definition's codes and scales
        vc, vs_exp = ref.cache_codes(ev.astype(np.float32))
        assert np.array_equal(vs[..., :vs_exp.shape[-1]], vs_exp)
        assert np.array_equal(V, vc * vs_exp.astype(np.float64).repeat(32, -1)[..., :D])
        # keys: scales within a step of 7 bits of the definition's, values within half a step (and what 32 bits are off)
        _, ks_exp = ref.cache_codes(ek.astype(np.float32))
        ks = ks[..., :ks_exp.shape[-1]].astype(np.float64)
        assert (np.abs(ks - ks_exp) <= 2.0 ** -6 * ks).all() and (ks == ks_exp).mean() > 0.99
        step = ks.repeat(32, -1)[..., :D]
        size = np.abs(ek).max() * 2
        assert (np.abs(K - ek) <= step * (0.5 + 7 * 2.0 ** -7) + (D / 2 + 8) * 2.0 ** -24 * size).all()  # (a scale rounded down: 7 steps fall short by 7 / 128 of one)
        # nothing else of the cache was touched
        others = np.setdiff1d(np.arange(pages * 64), slots)
        pl = ref.Places(D)
        b = host(cache)
        for at in (pl.k_byte, pl.v_byte):
            assert (b[others // 64, :][np.arange(len(others))[:, None, None], np.arange(G)[None, :, None], at[others % 64][:, None]] == 0x5A).all()
        # the same without asking for it back
        again = g.kv4_cache(pages, G, D)
        again.fill_(0x5A)
        q2 = g.qk_norm_rope(dev(c.x), H, G, D, **c.kwargs(interleaved), cache=again, slots=dev(slots))
        assert torch.equal(q, q2) and torch.equal(again, cache)


def test_slots_outside_the_cache_are_not_kept(g):
    c = _Case(6, 2, 2, 64, 64)
    cache = g.kv4_cache(2, 2, 64)
    cache.fill_(0x5A)
    slots = np.array([3, -1, 128, 2**31 - 1, -2**31, 127], np.int32)
    _, k, v = g.qk_norm_rope(dev(c.x), 2, 2, 64, **c.kwargs(False), cache=cache, slots=dev(slots), want_cached=True)
    kept = slots[[0, 5]]
    K, V, _, _ = _gather(host(cache), kept, 64)
    assert np.array_equal(host(k)[[0, 5]].astype(np.float64), K) and np.array_equal(host(v)[[0, 5]].astype(np.float64), V)
    alone = g.kv4_cache(2, 2, 64)
    alone.fill_(0x5A)
    c.x, c.pos, c.T = c.x[[0, 5]], c.pos[[0, 5]], 2
    g.qk_norm_rope(dev(c.x), 2, 2, 64, **c.kwargs(False), cache=alone, slots=dev(kept))
    assert torch.equal(alone, cache)


def test_positions_outside_the_table_take_its_ends(g):
    c = _Case(4, 2, 1, 64, 64)
    c.pos = np.array([-5, 2**31 - 1, 50, -2**31], np.int32)
    q, k = g.qk_norm_rope(dev(c.x), 2, 1, 64, **c.kwargs(False))
    c.pos = np.array([0, 49, 49, 0], np.int32)
    q2, k2 = g.qk_norm_rope(dev(c.x), 2, 1, 64, **c.kwargs(False))
    assert torch.equal(q, q2) and torch.equal(k, k2)


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_values_without_a_code(g, dtype):
    """NaN and infinities, zeros, tiny and huge groups through the cache's quantiser (no norm, no rotation: keys as they are)"""
    T, G, D = 5, 1, 64
    x = np.random.default_rng(1).standard_normal((T, 3 * D)).astype(dtype)
    x[0, D:D + 32] = 0
    x[1, D + 3], x[1, D + 40], x[2, 2 * D + 5] = np.nan, np.inf, -np.inf
    x[3, D:] *= dtype(1e-6)
    x[4, D:] *= dtype(2e4)
    cache = g.kv4_cache(1, G, D)
    _, k, v = g.qk_norm_rope(dev(x), 1, 1, D, norm=False, cache=cache, slots=dev(np.arange(T, dtype=np.int32)), want_cached=True)
    for got, part in ((k, x[:, D:2 * D]), (v, x[:, 2 * D:])):
        c, s = ref.cache_codes(part.astype(np.float32))
        assert np.array_equal(host(got)[:, 0].astype(np.float64), c * s.astype(np.float64).repeat(32, -1))
    # a vector with a value that is no number has no norm, and that is its head's alone (in fp16 2e4 times a value may be infinite)
    q, k = g.qk_norm_rope(dev(x), 1, 1, D)
    numbers = np.isfinite(x[:, D:2 * D].astype(np.float32)).all(1)
    assert np.isfinite(host(q)).all() and numbers[[0, 2, 3]].all() and not numbers[1]
    assert np.array_equal(np.isfinite(host(k)[:, 0]).all(1), numbers) and np.isnan(host(k)[1]).all()


def test_refusals(g):
    x = torch.zeros((4, 8 * 64), dtype=torch.float16, device="cuda")
    tab = torch.zeros((9, 32), device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    cache, slots = g.kv4_cache(1, 2, 64), torch.arange(4, dtype=torch.int32, device="cuda")
    assert g.qk_norm_rope(x, 4, 2, 64, cos=tab, sin=tab, positions=pos, cache=cache, slots=slots).shape == (4, 4, 64)
    for bad in (lambda: g.qk_norm_rope(x.half().cpu(), 4, 2, 64), lambda: g.qk_norm_rope(x, 5, 2, 64), lambda: g.qk_norm_rope(x.to(torch.int8), 4, 2, 64),
                lambda: g.qk_norm_rope(x, 4, 2, 64, q_weight=torch.ones(32, device="cuda")), lambda: g.qk_norm_rope(x, 4, 2, 64, cos=tab, sin=tab[:8], positions=pos),
                lambda: g.qk_norm_rope(x, 4, 2, 64, cos=tab, sin=tab), lambda: g.qk_norm_rope(x, 4, 2, 64, cos=tab, sin=tab, positions=pos[:3]),
                lambda: g.qk_norm_rope(x, 4, 2, 64, cos=tab, sin=tab, positions=pos.long()), lambda: g.qk_norm_rope(x, 4, 2, 64, cache=cache),
                lambda: g.qk_norm_rope(x, 4, 2, 64, cache=cache, slots=slots[:2]), lambda: g.qk_norm_rope(x, 4, 2, 64, cache=g.kv4_cache(1, 2, 128), slots=slots),
                lambda: g.qk_norm_rope(x.t(), 4, 2, 64)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(g.GpusqError):
        g.qk_norm_rope(x, 3, 2, 64)  # heads are no multiple of kv_heads
    with pytest.raises(g.GpusqError):
        g.qk_norm_rope(x, 4, 2, 60)
    with pytest.raises(g.GpusqError):
        g.qk_norm_rope(x, 4, 2, 64, cos=tab[:, :6].contiguous(), sin=tab[:, :6].contiguous(), positions=pos)  # 12 channels
    with pytest.raises(g.GpusqError):
        g.qk_norm_rope(x, 4, 2, 64, eps=-1.0)
    with pytest.raises(g.GpusqError):
        g.kv4_cache(3, 2, 260)


def test_one_token_whose_row_has_no_stride(g):
    """A column turned over: one contiguous row whose stride from token to token is 1"""
    c = _Case(1, 4, 2, 64, 64)
    q, k = g.qk_norm_rope(dev(c.x.reshape(-1, 1)).t(), 4, 2, 64, **c.kwargs(False))
    q0, k0 = g.qk_norm_rope(dev(c.x), 4, 2, 64, **c.kwargs(False))
    assert torch.equal(q, q0) and torch.equal(k, k0)
