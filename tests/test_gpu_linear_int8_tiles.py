"""The kernel of 8-bit layers for many tokens, by every kind of tile that it has (test_linear8_plans.py says which size takes which), against the definition in 64
bits; outputs and weights beyond 32-bit offsets."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_linear_int8_tokens import F16, F32, _check, _layer, _run
from test_gpu_parity import dev, g, host  # noqa: F401
from test_linear8_plans import SIZES

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", sorted(SIZES))
def test_tiles(g, M, N, K):
    """Every element, for both outputs, with and without GELU and a bias; nothing behind the last row; twice the same"""
    X, Wq, ws, bias = _layer(M, K, N, M + N + K)
    on = [dev(t) for t in (X, Wq, ws, bias)]
    for b, gelu, dts in ((bias, False, (F16, F32)), (None, False, (F32,)), (bias, True, (F16, F32))):
        exp, off = drafts.tokens8(X, Wq, ws, b, gelu)
        for dt in dts:
            whole = torch.full((M + 40, N), 7.0, dtype=dt, device="cuda")
            call = lambda out: g.linear_int8_tokens(on[0], on[1], on[2], bias=None if b is None else on[3], gelu=gelu, out_dtype=dt, out=out)  # noqa: E731
            call(whole[:M])
            _check(host(whole[:M]), exp, off)
            assert (whole[M:] == 7).all()
            assert torch.equal(call(torch.empty_like(whole[:M])), whole[:M])


def test_a_rows_result_does_not_depend_on_the_tile_it_lies_in(g):
    """To the bit (sums are exact): rows by themselves, in tiles of 64, 128 and 256 channels, beside few rows and many"""
    M, N, K = 1000, 16388, 336
    X, Wq, ws, bias = _layer(M, K, N, 4)
    for gelu, dt in ((True, F16), (False, F32)):
        whole = _run(g, X, Wq, ws, bias, gelu, dt)
        for a, b in ((0, 1), (3, 19), (100, 133), (200, 300), (500, 757), (999, 1000)):
            assert torch.equal(_run(g, X[a:b], Wq, ws, bias, gelu, dt), whole[a:b])
        for n in (260, 2052, 8196):
            assert torch.equal(_run(g, X, Wq[:n], ws[:n], bias[:n], gelu, dt), whole[:, :n])


@pytest.mark.parametrize("dt", [F16, F32])
def test_tiles_replayed_from_a_graph(g, dt):
    """Several tiles a workgroup, other tokens in each replay, eager work between them"""
    M, N, K = 1000, 16388, 336
    layers = [_layer(M, K, N, s)[0] for s in range(3)]
    _, Wq, ws, bias = _layer(M, K, N, 0)
    Wq, ws, bias, xs = dev(Wq), dev(ws), dev(bias), [dev(x) for x in layers]
    eager = [g.linear_int8_tokens(x, Wq, ws, bias=bias, gelu=True, out_dtype=dt) for x in xs]
    buf, graph = xs[0].clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = g.linear_int8_tokens(buf, Wq, ws, bias=bias, gelu=True, out_dtype=dt)
    for i in (1, 2, 0, 1):
        buf.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[i])
        y.zero_()


def test_outputs_beyond_32_bit_offsets(g):
    """4.6 GB of results: rows at its ends, in front of and behind 2^31 and 2^32 bytes"""
    M, N, K = 70001, 16388, 64
    X, Wq, ws, bias = _layer(M, K, N, 2)
    y = _run(g, X, Wq, ws, bias, False, F32)
    at = sorted({r for place in (0, 2**31, 2**32, 4 * M * N - 1) for r in range(place // (4 * N) - 2, place // (4 * N) + 3) if 0 <= r < M} | set(range(17, M, 7001)))
    _check(host(y[at]), *drafts.tokens8(X[at], Wq, ws, bias, False))


@pytest.mark.parametrize("M", [1, 20, 100])
def test_weights_beyond_32_bit_offsets(g, M):
    """4.3 GB of weights: channels at its ends, in front of and behind 2^31 and 2^32 bytes"""
    N, K = 33000, 131072
    gen = torch.Generator(device="cuda").manual_seed(M)
    Wq = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda", generator=gen)
    X, _, _, _ = _layer(M, K, 4, M)
    ws = (np.random.default_rng(M).uniform(0.5, 2, N) * 1e-4).astype(np.float32)
    y = g.linear_int8_tokens(dev(X), Wq, dev(ws), out_dtype=F32)
    at = sorted({c for place in (0, 2**31, 2**32, N * K - 1) for c in range(place // K - 3, place // K + 4) if 0 <= c < N} | set(range(11, N, 3001)))
    _check(host(y[:, at]), *drafts.tokens8(X, host(Wq[at]), ws[at], None, False))
