"""Linear layers on 4-bit weights with group scales against their definition in 64 bits."""
import numpy as np
import pytest

import decoder_reference as ref
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _weights(N, K, group, seed):
    r = np.random.default_rng(seed)
    codes = r.integers(-8, 8, (N, K)).astype(np.int8)
    scales = (r.uniform(0.5, 2, (N, K // group)) * 0.01).astype(np.float16)
    return codes, scales


def _gelu(x):
    from scipy.special import ndtr
    return x * ndtr(x)


def _check(y, X, codes, scales, group, bias, gelu, K):
    W = codes.astype(np.float64) * scales.astype(np.float64).repeat(group, 1)
    X64 = X.astype(np.float64)
    exp, size = X64 @ W.T, np.abs(X64) @ np.abs(W.T)
    if bias is not None:
        exp, size = exp + bias, size + np.abs(bias)
    # sums of K products in 32 bits, each step off by 2^-24 of what it has; GELU's slope is at most 1.13, its own error a few 2^-24
    off = (K + 16) * 2.0 ** -24 * size * (1.13 if gelu else 1)
    if gelu:
        exp = _gelu(exp)
        off = off + 2.0 ** -20 * np.abs(exp) + 1e-30
    if y.dtype == np.float16:
        off = off + 2.0 ** -11 * (np.abs(exp) + off) + 2.0 ** -25
    else:
        off = off + 2.0 ** -24 * np.abs(exp)
    assert (np.abs(y.astype(np.float64) - exp) <= off).all(), np.max(np.abs(y - exp) / off)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(4, 128), (37, 256), (130, 1152)])
def test_quantise_and_pack(g, N, K, group):
    r = np.random.default_rng(N + group)
    W = (r.standard_normal((N, K)) * 0.02).astype(np.float32)
    W[0, :group] = 0.0
    W[1, 3], W[2, 5], W[2, group - 1] = np.inf, np.nan, -3.0
    W[3, :group] = 1e-9  # a scale that is 0 in fp16
    W[-1, -group:] *= np.float32(1e-4)  # a scale among fp16's subnormal numbers
    codes, scales = g.quantize_groups_int4(dev(W), group)
    exp_c, exp_s = ref.groups_int4(W, group)
    assert np.array_equal(host(codes), exp_c) and np.array_equal(host(scales).view(np.uint16), exp_s.view(np.uint16))
    codes[0, 1] = -8  # not a code of the quantiser, but one of 4 bits
    exp_c[0, 1] = -8
    packed = g.pack_int4_groups(codes, scales, group)
    assert np.array_equal(host(packed), ref.pack_int4(exp_c, exp_s, group))


# a row, one more and one less than a block of 16, several, and more than one pass over the weights; fewer channels than a tile, tiles that
# are not full; K of one chunk of 32, of part of a step, of fewer and of more steps than wavefronts
@pytest.mark.parametrize("M", [1, 2, 7, 15, 16, 17, 32, 33, 48, 64, 65, 150])
@pytest.mark.parametrize("N,K,group", [(4, 32, 32), (20, 160, 32), (64, 192, 64), (1000, 1152, 128), (132, 1088, 64), (48, 2560, 128)])
def test_product(g, M, N, K, group):
    codes, scales = _weights(N, K, group, M + N)
    r = np.random.default_rng(M)
    X, bias = r.standard_normal((M, K)).astype(np.float16), r.standard_normal(N).astype(np.float32)
    packed = g.pack_int4_groups(dev(codes), dev(scales), group)
    for use_bias, gelu, dt in ((True, False, torch.float16), (False, False, torch.float32), (True, True, torch.float16), (True, True, torch.float32)):
        y = g.linear_int4(dev(X), packed, N, group, bias=dev(bias) if use_bias else None, gelu=gelu, out_dtype=dt)
        _check(host(y), X, codes, scales, group, bias if use_bias else None, gelu, K)


# K beyond what a wavefront keeps of its rows at once, for each number of rows, and at the edges of what it keeps
@pytest.mark.parametrize("M", [1, 16, 17, 33])
@pytest.mark.parametrize("K,group", [(2048, 128), (2112, 64), (4096, 32), (4224, 128), (6144, 64), (6176, 32), (8192, 32), (8320, 128), (16512, 64)])
def test_long_rows(g, M, K, group):
    N = 36
    codes, scales = _weights(N, K, group, M + K)
    r = np.random.default_rng(M)
    X, bias = r.standard_normal((M, K)).astype(np.float16), r.standard_normal(N).astype(np.float32)
    packed = g.pack_int4_groups(dev(codes), dev(scales), group)
    for gelu, dt in ((False, torch.float16), (True, torch.float32)):
        y = g.linear_int4(dev(X), packed, N, group, bias=dev(bias), gelu=gelu, out_dtype=dt)
        _check(host(y), X, codes, scales, group, bias, gelu, K)


# so many channels that a workgroup has several tiles of them; more than LDS has sums for
@pytest.mark.parametrize("M,N,K,group", [(1, 12308, 256, 128), (17, 12308, 160, 32), (3, 4500, 8448, 128), (40, 33000, 2176, 64)])
def test_many_channels(g, M, N, K, group):
    r = np.random.default_rng(M)
    codes = r.integers(-8, 8, (N, K), dtype=np.int8)
    scales = (r.uniform(0.5, 2, (N, K // group)) * 0.01).astype(np.float16)
    X, bias = r.standard_normal((M, K)).astype(np.float16), r.standard_normal(N).astype(np.float32)
    y = host(g.linear_int4(dev(X), g.pack_int4_groups(dev(codes), dev(scales), group), N, group, bias=dev(bias)))
    some = np.unique(np.concatenate([np.arange(20), r.integers(0, N, 400), np.arange(N - 200, N)]))
    _check(y[:, some], X, codes[some], scales[some], group, bias[some], False, K)


@pytest.mark.parametrize("dt", [torch.float16, torch.float32])
def test_gelu_of_large_values(g, dt):
    """Far beyond where it is the identity or 0, and infinite"""
    N, K = 8, 32
    codes = np.ones((N, K), np.int8)
    packed = g.pack_int4_groups(dev(codes), dev(np.ones((N, 1), np.float16)), 32)
    X = np.zeros((6, K), np.float16)
    X[:, 0] = 30000, -30000, 12, -12, np.inf, 0
    y = host(g.linear_int4(dev(X), packed, N, 32, gelu=True, out_dtype=dt)).astype(np.float64)  # (1e-30 in fp16 would be 0)
    assert (y[0] == 30000).all() and (y[1] == 0).all() and (y[2] == 12).all() and (np.abs(y[3]) < 1e-30).all() and (y[4] == np.inf).all() and (y[5] == 0).all()


def test_scales_of_every_size(g):
    """subnormal, huge and zero scales: the sums of a group meet them in 32 bits"""
    N, K, group = 32, 512, 32
    codes, scales = _weights(N, K, group, 3)
    scales[0], scales[1], scales[2, ::2], scales[3] = 6e-8, 5e-6, 0.0, 60000.0
    X = np.random.default_rng(4).standard_normal((9, K)).astype(np.float16)
    y = g.linear_int4(dev(X), g.pack_int4_groups(dev(codes), dev(scales), group), N, group, out_dtype=torch.float32)
    _check(host(y), X, codes, scales, group, None, False, K)


def test_a_row_without_a_value_keeps_to_itself(g):
    N, K, group = 52, 416, 32
    codes, scales = _weights(N, K, group, 5)
    packed = g.pack_int4_groups(dev(codes), dev(scales), group)
    X = np.random.default_rng(6).standard_normal((20, K)).astype(np.float16)
    clean = host(g.linear_int4(dev(X), packed, N, group))
    X[4, 7], X[18, 400] = np.nan, np.inf
    y = host(g.linear_int4(dev(X), packed, N, group))
    rest = [i for i in range(20) if i not in (4, 18)]
    assert np.array_equal(y[rest], clean[rest]) and np.isnan(y[4]).all() and not np.isfinite(y[18]).any()


def test_rows_of_a_larger_call_and_other_streams(g):
    """Every row as in a call of its own size, on a stream that is not the default one, outputs given"""
    N, K, group = 256, 1024, 64
    codes, scales = _weights(N, K, group, 7)
    packed = g.pack_int4_groups(dev(codes), dev(scales), group)
    X16 = np.random.default_rng(8).standard_normal((16, K)).astype(np.float16)
    X = dev(X16)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        out = torch.full((16, N), 7, dtype=torch.float16, device="cuda")
        assert g.linear_int4(X, packed, N, group, out=out) is out
        one = [g.linear_int4(X[i:i + 1], packed, N, group) for i in range(16)]
        torch.cuda.current_stream().synchronize()
    _check(host(out), X16, codes, scales, group, None, False, K)
    _check(host(torch.cat(one)), X16, codes, scales, group, None, False, K)


def test_refusals(g):
    packed = torch.zeros(g.lib().gpusq_int4_groups_packed_bytes(64, 128, 32), dtype=torch.uint8, device="cuda")
    X = torch.zeros((2, 128), dtype=torch.float16, device="cuda")
    assert g.linear_int4(X, packed, 64, 32).shape == (2, 64)
    for bad in (lambda: g.linear_int4(X.float(), packed, 64, 32), lambda: g.linear_int4(X, packed[:-16], 64, 32), lambda: g.linear_int4(X, packed, 68, 128),
                lambda: g.linear_int4(X, packed, 64, 32, bias=torch.zeros(63, device="cuda")), lambda: g.linear_int4(X.cpu(), packed, 64, 32),
                lambda: g.linear_int4(X[:, ::2], packed, 64, 32), lambda: g.linear_int4(X, packed, 64, 32, out=torch.zeros((2, 64), device="cuda")),
                lambda: g.quantize_groups_int4(X, 32), lambda: g.pack_int4_groups(X.to(torch.int8), torch.zeros((2, 3), dtype=torch.float16, device="cuda"), 32)):
        with pytest.raises(ValueError):
            bad()
    for group in (16, 0, 48):
        with pytest.raises(g.GpusqError):
            g.quantize_groups_int4(X.float(), group)
    with pytest.raises(g.GpusqError):
        g.quantize_groups_int4(torch.zeros((2, 100), device="cuda"), 32)


# steps of K that the wavefronts do not deal out evenly: behind the last one some have none
@pytest.mark.parametrize("M", [1, 20, 40])
@pytest.mark.parametrize("K", [128, 1152, 2176, 8320])
def test_an_infinite_scale(g, M, K):
    """The last group of a channel with a scale that is infinite: its sum, which is not 0, times it, in that channel alone"""
    N, group = 20, 32
    codes, scales = _weights(N, K, group, 8)
    codes[:, -group:] = 1
    X = np.abs(np.random.default_rng(9).standard_normal((M, K))).astype(np.float16) + np.float16(0.5)
    clean = host(g.linear_int4(dev(X), g.pack_int4_groups(dev(codes), dev(scales), group), N, group, out_dtype=torch.float32))
    scales[5, -1], scales[7, -1] = np.inf, -np.inf
    y = host(g.linear_int4(dev(X), g.pack_int4_groups(dev(codes), dev(scales), group), N, group, out_dtype=torch.float32))
    assert (y[:, 5] == np.inf).all() and (y[:, 7] == -np.inf).all()
    others = [n for n in range(N) if n not in (5, 7)]
    assert np.array_equal(y[:, others], clean[:, others])
