"""8-bit layers for 17 to 64 tokens where whole rows of weights and tiles meet: either side of each border, by element, and the same to the bit."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_linear_int8_tokens import F16, F32, _check, _layer, _run
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [32, 33, 64, 65])
@pytest.mark.parametrize("N", [8188, 8192, 8196, 12284, 12288, 12292])
@pytest.mark.parametrize("K", [1024, 2048, 2064, 4096, 4112])
def test_borders(g, M, N, K):
    X, Wq, ws, bias = _layer(M, K, N, M + N + K)
    y = _run(g, X, Wq, ws, bias, False, F32)
    _check(host(y), *drafts.tokens8(X, Wq, ws, bias, False))
    # channels and rows by themselves, which another kernel takes
    assert torch.equal(_run(g, X, Wq[:100], ws[:100], bias[:100], False, F32), y[:, :100])
    assert torch.equal(_run(g, X[:17], Wq, ws, bias, False, F32), y[:17])
    exp, off = drafts.tokens8(X, Wq, ws, bias, True)
    _check(host(_run(g, X, Wq, ws, bias, True, F16)), exp, off)
    assert np.isfinite(exp).all()
