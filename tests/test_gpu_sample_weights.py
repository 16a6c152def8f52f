"""How well small weights of sample_tokens are known: by the shares of tokens that only a random number of 0 draws."""
import numpy as np
import pytest

from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = np.float32


@pytest.mark.parametrize("T", [1.0, 0.37, 2.5])
@pytest.mark.parametrize("parts", [False, True])
def test_shares_of_small_weights(g, T, parts):
    """Of two tokens the first is drawn by 0, whatever its weight is: 2^-30 of it and 2^-45 of the greatest's, and the share's own rounding to 32 bits.  (In a row over
    several workgroups the greatest lies in another one's part)"""
    rows, V = (32, 70000) if parts else (4096, 2)
    T = F32(T)
    x = np.full((rows, V), -np.inf, F32)
    x[:, -1] = np.random.default_rng(1).uniform(-3, 3, rows)
    x[:, 0] = x[:, -1] - (np.linspace(0.01, 27.72, rows) * np.float64(T)).astype(F32)
    tokens, probs = (host(t) for t in g.sample_tokens(dev(x), dev(np.zeros(rows, F32)), temperature=dev(np.full(rows, T))))
    w = np.exp((x[:, 0].astype(np.float64) - x[:, -1]) / np.float64(T))
    there = w > 2.0 ** -40 * (1 + 2.0 ** -20)  # (next to the border either)
    assert (tokens[there] == 0).all() and there.sum() >= rows - rows // 500 - 1
    share, got = (w / (1 + w))[there], probs[there].astype(np.float64)
    assert (np.abs(got - share) <= (2.0 ** -30 * share + 2.0 ** -45) * (1 + 2.0 ** -20) + 2.0 ** -24 * share).all()


def test_what_has_no_weight(g):
    """Below 2^-40, or so far from the greatest that 32 bits do not hold the difference, whatever the temperature"""
    x = np.array([[-27.8, 0.0], [-1e30, 1.0], [-3e38, 3e38], [-3e38, 3e38], [-65504, 65504]], F32)
    T = np.array([1, 1, 1, 1e38, np.inf], F32)
    tokens, probs = (host(t) for t in g.sample_tokens(dev(x), dev(np.zeros(5, F32)), temperature=dev(T)))
    assert tokens.tolist() == [1, 1, 1, 1, 0] and probs.tolist() == [1, 1, 1, 1, 0.5]
