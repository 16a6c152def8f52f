"""Attention of a tree of drafted tokens over the 4-bit cache, against the definition in 64 bits and what the kernels' own roundings allow."""
import numpy as np
import pytest

import decoder_reference as ref
import drafts_reference as drafts
from test_gpu_attention import HEADS, _Cache, _check
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _expected(c, q, counts, sets):
    """sets: for each new token the new ones that it sees"""
    out, off, at, H = np.zeros(q.shape), np.zeros(q.shape), 0, q.shape[1]
    for b, n in enumerate(counts):
        L = c.lens[b]
        seen = np.zeros((n, L), bool)
        seen[:, :max(L - n, 0)] = True
        for i in range(n):
            for j in sets[at + i]:
                if j < n and L - n + j >= 0:
                    seen[i, L - n + j] = True
        for h in range(H):
            out[at:at + n, h], off[at:at + n, h] = ref.attend(q[at:at + n, h].astype(np.float64), c.K[b][:, h * c.G // H], c.V[b][:, h * c.G // H], seen, c.D ** -0.5)
        at += n
    return out, off


def _run(g, c, q, counts, words, **kw):
    cu = np.r_[0, np.cumsum(counts)].astype(np.int32)
    return g.attention_kv4(dev(q), dev(c.pages), dev(c.table), dev(np.array(c.lens, np.int32)), cu_q=dev(cu), max_q=max(counts), tree=dev(words), **kw)


def _sets(r, counts, kind):
    sets = []
    for n in counts:
        if kind == "tree":
            t = [-1] + [int(r.integers(0, i)) for i in range(1, n)]
            sets += [drafts.chain(t, i) for i in range(n)]
        else:  # any bits: nodes behind, not itself, none at all
            sets += [np.nonzero(r.random(n) < r.choice([0.0, 0.3, 1.0]))[0].tolist() for _ in range(n)]
    return sets


# few columns and many; lengths at the edges of tiles and pages; trees that are the whole history or more than it; nodes in several words that begin
# anywhere in a tile; bits behind the last node are not read
@pytest.mark.parametrize("H,G,D", HEADS)
@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("lens,counts", [([1, 40, 33, 64, 70], [1, 3, 2, 4, 1]), ([40, 7, 5, 130, 3, 200, 64], [2, 1, 5, 35, 6, 70, 64]), ([300, 65], [97, 33])])
def test_trees(g, H, G, D, kind, lens, counts):
    r = np.random.default_rng(H + sum(lens))
    c = _Cache(lens, G, D, seed=4)
    q = r.standard_normal((sum(counts), H, D)).astype(np.float16)
    sets = _sets(r, counts, kind)
    W = -(-max(counts) // 32) + (1 if kind == "any" else 0)
    words = drafts.bits(sets, W)
    if kind == "any":  # bits of nodes that are none
        n = np.repeat(counts, counts)
        for i in range(len(words)):
            for j in range(n[i], 32 * W):
                words[i, j // 32] |= np.int32(np.uint32(1 << j % 32).view(np.int32)) if r.random() < 0.5 else 0
    exp, off = _expected(c, q, counts, sets)
    y = _run(g, c, q, counts, words)
    _check(y, exp, off)
    # rows that see nothing are 0
    empty = off.max(-1) == 2.0 ** -24
    assert not host(y)[empty].any()


@pytest.mark.parametrize("H,G,D,L,n", [(8, 2, 64, 5000, 9), (4, 1, 128, 9001, 4), (8, 1, 128, 3000, 63), (4, 2, 80, 20001, 3), (2, 1, 256, 2500, 40)])
def test_long_histories_are_cut_and_joined(g, H, G, D, L, n):
    """The tree may lie across two parts, or in the last one alone"""
    r = np.random.default_rng(L)
    c = _Cache([L, 70], G, D, seed=2)
    counts = [n, min(n, 30)]
    size = g.lib().gpusq_attention_tree_kv4_workspace_bytes(sum(counts), 2, n, c.table.shape[1], H, G, D)
    assert size > 0
    q = r.standard_normal((sum(counts), H, D)).astype(np.float16)
    sets = _sets(r, counts, "tree")
    words = drafts.bits(sets, -(-n // 32))
    y = _run(g, c, q, counts, words)
    _check(y, *_expected(c, q, counts, sets))
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # NaN
    assert torch.equal(_run(g, c, q, counts, words, workspace=ws, out=torch.full_like(y, 7)), y)


def test_a_chain_is_causal_attention(g):
    """To the bit where both have the same kernel (few columns): the same products in the same order, and the same keys hidden.  Else either is the definition,
    within what its roundings allow"""
    r = np.random.default_rng(6)
    for (H, G, D), counts in (((8, 2, 128), [3, 1]), ((6, 2, 80), [40, 21]), ((4, 4, 64), [9, 70])):
        lens = [200, 90]
        c = _Cache(lens, G, D, seed=7)
        q = r.standard_normal((sum(counts), H, D)).astype(np.float16)
        sets = [list(range(i + 1)) for n in counts for i in range(n)]
        cu = dev(np.r_[0, np.cumsum(counts)].astype(np.int32))
        plain = g.attention_kv4(dev(q), dev(c.pages), dev(c.table), dev(np.array(lens, np.int32)), cu_q=cu, max_q=max(counts))
        tree = _run(g, c, q, counts, drafts.bits(sets, -(-max(counts) // 32)))
        if max(counts) * H // G <= 16:
            assert torch.equal(tree, plain)
        else:
            exp = _expected(c, q, counts, sets)
            _check(tree, *exp)
            _check(plain, *exp)


# blocks of 2, 3 and 4 times 16 columns, 4 or 8 wavefronts, up to 256 columns of many pairs (beyond 192 of few: another kernel)
@pytest.mark.parametrize("B,H,G,D,n", [(70, 16, 4, 128, 12), (130, 8, 4, 128, 14), (140, 16, 4, 128, 11), (130, 8, 4, 64, 13), (140, 8, 4, 64, 20), (130, 8, 4, 64, 25), (20, 4, 1, 128, 62),
                                       (3, 4, 1, 128, 48), (3, 4, 1, 128, 49), (18, 4, 1, 64, 64), (18, 4, 1, 64, 65), (17, 2, 1, 256, 20)])
def test_batches_of_trees(g, B, H, G, D, n):
    r = np.random.default_rng(B * n)
    counts = [n] + r.integers(1, n + 1, B - 1).tolist()
    lens = [c + int(r.integers(0, 140)) for c in counts]
    c = _Cache(lens, G, D, seed=12)
    q = r.standard_normal((sum(counts), H, D)).astype(np.float16)
    sets = _sets(r, counts, "tree")
    words = drafts.bits(sets, -(-n // 32))
    y = _run(g, c, q, counts, words)
    _check(y, *_expected(c, q, counts, sets))
    assert torch.equal(_run(g, c, q, counts, words), y)


def test_pages_that_are_none_and_what_is_no_number(g):
    """A page number outside the cache is not seen; a query that is no number is NaN where it sees a key, 0 where it sees none; hidden keys hold NaN"""
    r = np.random.default_rng(9)
    H, G, D, n = 2, 1, 64, 5
    for counts in ([n], [n + 40]):
        n = counts[0]
        c = _Cache([64 + n], G, D, seed=9)  # the second page holds the tree
        words = drafts.bits([[i] for i in range(n)], -(-n // 32))
        words[1] = 0
        q = r.standard_normal((n, H, D)).astype(np.float16)
        table = c.table.copy()
        table[0, 1] = 2**30  # the tree is in no page
        lens, cu = dev(np.array(c.lens, np.int32)), dev(np.array([0, n], np.int32))
        call = lambda q, table, lens: host(g.attention_kv4(dev(q), dev(c.pages), dev(table), lens, cu_q=cu, max_q=n, tree=dev(words)))  # noqa: E731
        exp, off = _expected(c, q, [n], [[] for _ in range(n)])
        assert (np.abs(call(q, table, lens) - exp) <= off).all()
        # no history: only the tree's own bits
        table = c.table[:, 1:].copy()
        q[:2] = np.nan
        y = call(q, table, dev(np.array([n], np.int32)))
        assert np.isnan(y[0]).all() and (y[1] == 0).all() and np.isfinite(y[2:]).all()
        V = c.V[0][64:, 0]
        assert (np.abs(y[2:] - V[2:n, None]) <= 2.0 ** -10 * np.abs(V[2:n, None]) + 2.0 ** -24).all()  # one key each: its value


# few columns, blocks of 2 and 3, the kernel for many; heads of every padding
@pytest.mark.parametrize("H,G,D,L,n", [(4, 4, 64, 30, 9), (8, 2, 128, 300, 4), (8, 2, 128, 3000, 12), (4, 1, 80, 70, 40), (3, 1, 40, 64, 33), (2, 2, 136, 100, 12), (7, 1, 256, 90, 30), (8, 1, 128, 500, 40),
                                       (16, 1, 64, 200, 30)])
def test_nodes_that_are_no_numbers(g, H, G, D, L, n):
    """Keys and values of some nodes with a scale that is infinite, or a value that is none: who sees one is NaN, of that head; nobody else notices"""
    r = np.random.default_rng(L + n)
    c = _Cache([L + n], G, D, seed=5)
    pl = ref.Places(D)
    sets = _sets(r, [n], "tree")
    groups = -(-D // 32)
    poisoned = {int(n // 2): [(pl.v_scale, groups - 1, 0x7C00)], n - 1: [(pl.v_scale, 0, 0x7E00)], n // 3: [(pl.k_scale, 0, 0x7C00)], 1: [(pl.v_scale, 0, 0xFC00), (pl.k_scale, groups - 1, 0x7E01)]}
    head = G - 1  # the others' are as they were
    for node, places in poisoned.items():
        t = L + node
        halves = c.pages[c.table[0, t // 64]].view(np.uint16)
        for at, group, bits in places:
            place = at[t % 64, group]
            halves[head, place] = bits
        c.K[0][t, head] = c.V[0][t, head] = 0
    q = r.standard_normal((n, H, D)).astype(np.float16)
    words = drafts.bits(sets, -(-n // 32))
    y = host(_run(g, c, q, [n], words)).astype(np.float64)
    exp, off = _expected(c, q, [n], sets)
    sees = np.array([any(j in poisoned for j in nodes) for nodes in sets])
    of_head = np.arange(H) * G // H == head
    wrong = sees[:, None] & of_head[None]
    assert sees.any() and not sees.all()
    assert np.isnan(y[wrong]).all()
    assert (np.abs(y - exp) <= off)[~wrong].all()


def test_replayed_from_a_graph(g):
    r = np.random.default_rng(11)
    H, G, D, counts = 8, 2, 128, [7, 12]
    c = _Cache([3000, 150], G, D, seed=3)
    q, cu, lens = dev(r.standard_normal((19, H, D)).astype(np.float16)), dev(np.array([0, 7, 19], np.int32)), dev(np.array(c.lens, np.int32))
    pages, table = dev(c.pages), dev(c.table)
    words = [dev(drafts.bits(_sets(r, counts, "tree"), 1)) for _ in range(3)]
    tree, graph = words[0].clone(), torch.cuda.CUDAGraph()
    call = lambda t: g.attention_kv4(q, pages, table, lens, cu_q=cu, max_q=12, tree=t)  # noqa: E731
    eager = [call(w) for w in words]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = call(tree)
    for i in (1, 2, 0, 1):
        tree.copy_(words[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i])


def test_refusals(g):
    q, cache = torch.zeros((4, 4, 64), dtype=torch.float16, device="cuda"), g.kv4_cache(2, 2, 64)
    table, lens = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    tree = torch.zeros((4, 1), dtype=torch.int32, device="cuda")
    for bad in (tree[:3], tree.long(), tree[:, 0], tree.cpu()):
        with pytest.raises(ValueError):
            g.attention_kv4(q, cache, table, lens, max_q=4, tree=bad)
    q = torch.zeros((33, 4, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(g.GpusqError) as e:
        g.attention_kv4(q, cache, table, lens, max_q=33, tree=torch.zeros((33, 1), dtype=torch.int32, device="cuda"))
    assert e.value.status == g.ERR_SHAPE
