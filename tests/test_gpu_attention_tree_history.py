"""Trees of drafted tokens behind a history with scales that are no finite numbers: every node sees the history, so every node notices."""
import numpy as np
import pytest

import decoder_reference as ref
import drafts_reference as drafts
from test_gpu_attention import _Cache, _check
from test_gpu_attention_tree import _expected, _run, _sets
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# The history ends at the edges of a tile of 32 or 64 keys and within either half of one; few columns, blocks of 2 and 3, the kernel for many columns (more
# than 192 of few pairs, of heads beyond 128 more than 32); heads of every padding
@pytest.mark.parametrize("H,G,D,n", [(4, 4, 64, 9), (8, 2, 128, 12), (8, 1, 64, 30), (16, 1, 128, 40), (9, 1, 80, 37), (16, 1, 64, 20), (2, 1, 256, 40), (14, 2, 136, 9)])
@pytest.mark.parametrize("L", [64, 95, 96, 97, 104, 127, 128, 160, 300])
def test_a_history_that_is_no_number(g, H, G, D, n, L):
    """One of its values' scales in the page's half that the tree does not reach, in the one that it does, or a page in front: the results of that group of
    32 channels are no finite numbers, in every node, as they are of causal attention over the same cache.  Other heads are as they were"""
    r = np.random.default_rng(L + n)
    pl = ref.Places(D)
    head, group = G - 1, (-(-D // 32)) - 1
    counts = [n]
    c = _Cache([L + n], G, D, seed=5)
    sets = _sets(r, counts, "tree")
    words = drafts.bits(sets, -(-n // 32))
    q = r.standard_normal((n, H, D)).astype(np.float16)
    exp, off = _expected(c, q, counts, sets)
    _check(_run(g, c, q, counts, words), exp, off)
    of_head = np.arange(H) * G // H == head
    whole = c.pages.copy()
    last = (L - 1) // 64 * 64
    for t in sorted({last + 5, min(last + 40, L - 1), L - 1, 3}):
        if t >= L:
            continue
        for place, bits in ((pl.v_scale[t % 64, group], 0x7C00), (pl.v_scale[t % 64, group], 0x7E01), (pl.k_scale[t % 64, group], 0xFC00)):
            c.pages = whole.copy()
            c.pages[c.table[0, t // 64]].view(np.uint16)[head, place] = bits
            y = host(_run(g, c, q, counts, words)).astype(np.float64)
            assert not np.isfinite(y[:, of_head, 32 * group:]).any(), (t, bits)
            assert (np.abs(y - exp) <= off)[:, ~of_head].all(), (t, bits)
            causal = host(g.attention_kv4(dev(q), dev(c.pages), dev(c.table), dev(np.array(c.lens, np.int32)), max_q=n)).astype(np.float64)
            assert not np.isfinite(causal[:, of_head, 32 * group:]).any(), (t, bits)


@pytest.mark.parametrize("L", [40, 63, 97])
def test_of_two_sequences_one_notices(g, L):
    """... and nodes of another sequence do not"""
    H, G, D, counts = 16, 1, 64, [30, 21]
    r = np.random.default_rng(L)
    c = _Cache([L + counts[0], L + counts[1]], G, D, seed=6)
    pl = ref.Places(D)
    sets = _sets(r, counts, "tree")
    words = drafts.bits(sets, 1)
    q = r.standard_normal((sum(counts), H, D)).astype(np.float16)
    exp, off = _expected(c, q, counts, sets)
    t = L // 64 * 64 + 7
    c.pages[c.table[0, t // 64]].view(np.uint16)[0, pl.v_scale[t % 64, 1]] = 0x7C00
    y = host(_run(g, c, q, counts, words)).astype(np.float64)
    assert not np.isfinite(y[:30, :, 32:]).any()
    assert (np.abs(y - exp) <= off)[30:].all()
