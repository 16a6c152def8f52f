"""Linear layers in 8-bit integers with scales for each token and channel, against their definition in 64 bits."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _layer(M, K, N, seed, x=np.float16):
    r = np.random.default_rng(seed)
    X = (r.standard_normal((M, K)) * r.uniform(0.01, 30, (M, 1))).astype(x)
    return X, r.integers(-128, 128, (N, K)).astype(np.int8), (r.uniform(0.5, 2, N) * 0.001).astype(np.float32), r.standard_normal(N).astype(np.float32)


def _check(y, exp, off):
    if y.dtype == np.float16:
        off = off + 2.0 ** -11 * (np.abs(exp) + off) + 2.0 ** -25
    assert (np.abs(y.astype(np.float64) - exp) <= off).all(), np.max(np.abs(y - exp) / off)


def _run(g, X, Wq, ws, bias, gelu, dt, **kw):
    return g.linear_int8_tokens(dev(X), dev(Wq), dev(ws), bias=None if bias is None else dev(bias), gelu=gelu, out_dtype=dt, **kw)


F16, F32 = torch.float16, torch.float32


# rows around blocks of 16, 32, 64 and tiles of 256; channels that fill no tile; K of a part of a step, of whole ones, of more than a kernel keeps
@pytest.mark.parametrize("M", [1, 2, 9, 16, 17, 31, 33, 64, 65, 130, 257])
@pytest.mark.parametrize("N,K", [(4, 16), (20, 48), (64, 64), (100, 208), (516, 1024), (132, 1104), (1000, 528), (36, 4112)])
def test_product(g, M, N, K):
    X, Wq, ws, bias = _layer(M, K, N, M + N + K)
    for b, gelu, dt in ((bias, False, F16), (None, False, F32), (bias, True, F16), (bias, True, F32)):
        _check(host(_run(g, X, Wq, ws, b, gelu, dt)), *drafts.tokens8(X, Wq, ws, b, gelu))


@pytest.mark.parametrize("M", [1, 5, 16, 20, 40, 70, 300])
@pytest.mark.parametrize("K", [2048, 2064, 8192, 8208, 16400, 32784])
def test_long_rows_of_fp32(g, M, K):
    N = 72
    X, Wq, ws, bias = _layer(M, K, N, M + K, np.float32)
    for dt in (F16, F32):
        _check(host(_run(g, X, Wq, ws, bias, False, dt)), *drafts.tokens8(X, Wq, ws, bias, False))


def test_the_longest_rows(g):
    """Every product as large as it may be: the sums come close to 32 bits"""
    K, N = 132096, 8
    X = np.full((18, K), 3.0, np.float16)
    X[1::2] = -3.0
    Wq = np.full((N, K), -128, np.int8)
    Wq[4:] = 127
    ws = np.full(N, 1e-6, np.float32)
    for M in (1, 18):
        _check(host(_run(g, X[:M], Wq, ws, None, False, F32)), *drafts.tokens8(X[:M], Wq, ws, None, False))


# many channels, several tiles a workgroup; many rows, tiles of every height
@pytest.mark.parametrize("M,N,K", [(1, 40004, 512), (13, 20500, 2048), (30, 12300, 1040), (61, 9000, 640), (100, 5000, 512), (700, 1540, 832), (1500, 776, 320), (2309, 2052, 192)])
def test_large(g, M, N, K):
    X, Wq, ws, bias = _layer(M, K, N, M + N)
    exp, off = drafts.tokens8(X, Wq, ws, bias, False)
    for dt in (F16, F32):
        _check(host(_run(g, X, Wq, ws, bias, False, dt)), exp, off)
    exp, off = drafts.tokens8(X, Wq, ws, bias, True)
    _check(host(_run(g, X, Wq, ws, bias, True, F16)), exp, off)


@pytest.mark.parametrize("M", [6, 40, 300])
def test_codes_are_the_quantisers(g, M):
    """Against quantize_int8 by rows and the products of the existing dense layer: rows of zeros, of one value, that are half-way between codes, with values
    that are no numbers, tiny ones"""
    K, N = 272, 64
    r = np.random.default_rng(M)
    X = r.standard_normal((M, K)).astype(np.float32)
    X[0] = 0
    X[1] = 1e-42  # (a scale that is subnormal)
    X[2, :128] = np.arange(128) - 0.5
    X[2, 128:] = 127
    X[3, 5] = np.nan
    X[4] = 0
    X[4, 271] = -7
    Wq = r.integers(-127, 128, (N, K)).astype(np.int8)
    ones = np.ones(N, np.float32)
    y = host(_run(g, X, Wq, ones, None, False, F32))
    q, s = (host(t) for t in g.quantize_int8(dev(X), g.PER_ROW))
    acc = q.astype(np.int64) @ Wq.T.astype(np.int64)
    assert np.array_equal(y, acc.astype(np.float32) * s[:, None])
    X[5, 0] = np.inf
    y = host(_run(g, X, Wq, ones, None, False, F32))
    assert np.isnan(y[5]).all() and np.isfinite(y[:5]).all()


def test_rows_are_independent(g):
    """A token's result does not depend on the others, nor on how many there are (to the bit: sums are exact)"""
    X, Wq, ws, bias = _layer(600, 528, 260, 9)
    whole = host(_run(g, X, Wq, ws, bias, True, F16))
    for a, b in ((0, 1), (7, 20), (100, 133), (200, 300), (1, 600)):
        assert np.array_equal(host(_run(g, X[a:b], Wq, ws, bias, True, F16)), whole[a:b])


@pytest.mark.parametrize("M", [3, 50, 400])
def test_workspace_output_and_graph(g, M):
    K, N = 336, 132
    layers = [_layer(M, K, N, s) for s in range(3)]
    Wq, ws, bias = (dev(t) for t in layers[0][1:])
    xs = [dev(layer[0]) for layer in layers]
    eager = [g.linear_int8_tokens(x, Wq, ws, bias=bias) for x in xs]
    size = g.lib().gpusq_linear_int8_tokens_workspace_bytes(M, K)
    w, out = torch.full((size,), 255, dtype=torch.uint8, device="cuda"), torch.full((M, N), 7.0, dtype=F16, device="cuda")
    assert g.linear_int8_tokens(xs[1], Wq, ws, bias=bias, workspace=w, out=out) is out and torch.equal(out, eager[1])
    buf, graph = xs[0].clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = g.linear_int8_tokens(buf, Wq, ws, bias=bias)
    for i in (1, 2, 0, 1):
        buf.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[i])


def test_behind_the_last_row_nothing_is_written(g):
    for M, N, K in ((1, 4, 16), (9, 20, 48), (33, 68, 80), (70, 260, 80), (300, 516, 144)):
        X, Wq, ws, _ = _layer(M, K, N, M)
        for dt in (F16, F32):
            whole = torch.full((M + 300, N), 7.0, dtype=dt, device="cuda")
            g.linear_int8_tokens(dev(X), dev(Wq), dev(ws), out=whole[:M], out_dtype=dt)
            assert (host(whole)[M:] == 7).all() and not (host(whole)[:M] == 7).all()


def test_refusals(g):
    X, W, s = torch.zeros((3, 32), dtype=F16, device="cuda"), torch.zeros((8, 32), dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda")
    for call in (lambda: g.linear_int8_tokens(X.double(), W, s), lambda: g.linear_int8_tokens(X, W[:, :16].contiguous(), s), lambda: g.linear_int8_tokens(X, W, s[:7]),
                 lambda: g.linear_int8_tokens(X, W, s, bias=s[:4]), lambda: g.linear_int8_tokens(X, W.float(), s), lambda: g.linear_int8_tokens(X.cpu(), W, s),
                 lambda: g.linear_int8_tokens(torch.zeros((3, 64), dtype=F16, device="cuda")[:, ::2], W, s), lambda: g.linear_int8_tokens(X, W, s, out=torch.zeros((3, 8), device="cuda")),
                 lambda: g.linear_int8_tokens(X, W, s, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    z = lambda *shape, dt=torch.int8: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    for call, status in ((lambda: g.linear_int8_tokens(z(3, 24, dt=F16), z(8, 24), s), g.ERR_UNSUPPORTED), (lambda: g.linear_int8_tokens(X, z(6, 32), s[:6].clone()), g.ERR_UNSUPPORTED),
                         (lambda: g.linear_int8_tokens(X, W, s, out_dtype=torch.int8), g.ERR_UNSUPPORTED), (lambda: g.linear_int8_tokens(z(1, 132112, dt=F16), z(8, 132112), s), g.ERR_SHAPE)):
        with pytest.raises(g.GpusqError) as e:
            call()
        assert e.value.status == status
