"""Trees of drafted tokens: what each follows, where it stands, and the branch that is kept, moved together in the caches.  Whole numbers: exact."""
import numpy as np
import pytest

import decoder_reference as ref
import drafts_reference as drafts
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _tree(r, n, kind):
    if kind == "chain":
        return np.arange(-1, n - 1)
    if kind == "star":
        return np.r_[-1, np.zeros(n - 1)].astype(int) if n else np.zeros(0, int)
    if kind == "comb":  # the even nodes a chain, an odd one behind each
        return np.array([-1 if i == 0 else i - 1 if i % 2 else i - 2 for i in range(n)], dtype=np.int64)
    if kind == "forest":  # several roots, parents that are none: themselves, nodes behind, numbers far off
        return np.array([r.choice([-1, i, i + 1, n + 7, -2**31, 2**31 - 1]) if r.random() < 0.3 else r.integers(0, i) if i else -1 for i in range(n)], dtype=np.int64)
    return np.array([-1] + [max(0, i - 1 - int(r.integers(0, i) * r.random())) for i in range(1, n)][:max(0, n - 1)])[:n]


def _batch(r, counts, kinds=("tree",), longest=300):
    trees = [_tree(r, n, kinds[b % len(kinds)]) for b, n in enumerate(counts)]
    lens = [n + int(r.integers(0, longest)) for n in counts]
    return trees, lens, np.r_[0, np.cumsum(counts)].astype(np.int32)


@pytest.mark.parametrize("counts", [[1], [2, 0, 5], [31, 32, 33], [64, 1, 7, 100], [0, 0, 3], [512, 40]])
@pytest.mark.parametrize("kinds", [("tree",), ("chain", "star"), ("forest",)])
def test_draft_tree(g, counts, kinds):
    r = np.random.default_rng(sum(counts))
    trees, lens, cu = _batch(r, counts, kinds)
    per = max(1, -(-max(lens) // 64))
    table = r.integers(0, 1000, (len(counts), per)).astype(np.int32)
    table[0, -1] = -5  # no page
    table[-1, 0] = 2**31 - 1
    n, W = max(counts), -(-max(counts) // 32)
    got = [host(t) for t in g.draft_tree(dev(np.concatenate(trees).astype(np.int32)), dev(np.array(lens, np.int32)), dev(table), cu_q=dev(cu), max_q=n)]
    for b, t in enumerate(trees):
        own, before = slice(cu[b], cu[b + 1]), lens[b] - len(t)
        chains = [drafts.chain(t, i) for i in range(len(t))]
        assert np.array_equal(got[0][own], drafts.bits(chains, W))
        assert np.array_equal(got[1][own], [before + len(c) - 1 for c in chains])
        assert np.array_equal(got[2][own], [drafts.slots(table[b], before + i) for i in range(len(t))])


def test_draft_tree_without_cu_and_what_it_leaves_alone(g):
    """As many tokens each; a history shorter than the new tokens, or none; more nodes than max_q; tokens that no sequence has"""
    r = np.random.default_rng(3)
    t = [_tree(r, 6, "tree") for _ in range(3)]
    lens, table = np.array([100, 4, -3], np.int32), np.array([[3, 9], [1, 2], [4, 5]], np.int32)
    a = [host(x) for x in g.draft_tree(dev(np.concatenate(t).astype(np.int32)), dev(lens), dev(table))]
    for b in range(3):
        before = max(int(lens[b]), 0) - 6
        assert np.array_equal(a[1][6 * b:6 * b + 6], [before + len(drafts.chain(t[b], i)) - 1 for i in range(6)])
        assert np.array_equal(a[2][6 * b:6 * b + 6], [drafts.slots(table[b], before + i) for i in range(6)])
    parents = dev(np.concatenate(t).astype(np.int32))
    tree, positions, slots = (torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((18, 1), (18,), (18,)))
    cu = dev(np.array([2, 8, 8, 13], np.int32))
    g.calls.gpusq_draft_tree(parents, dev(np.array([70, 5, 90], np.int32)), cu, dev(table), tree, positions, slots, 18, 3, 4, 2)
    p = host(parents)
    for s, e, l in ((2, 8, 70), (8, 13, 90)):
        for i in range(4):
            assert host(positions)[s + i] == l - (e - s) + len(drafts.chain(p[s:e], i)) - 1
        assert (host(positions)[s + 4:e] == 77).all() and (host(tree)[s + 4:e] == 77).all() and (host(slots)[s + 4:e] == 77).all()
    for x in (tree, positions, slots):
        assert (host(x)[:2] == 77).all() and (host(x)[13:] == 77).all()


def _tokens(r, trees, depth):
    """Drafts and drawn tokens with a branch that agrees for some nodes, and others that would, had their parents been kept or come first"""
    drafted, sampled = [], []
    for t in trees:
        n = len(t)
        d, s = r.integers(0, 3, n), r.integers(0, 3, n)  # (few tokens: children of the same parent with the same draft)
        at = 0
        for _ in range(depth):
            follow = [i for i in range(at + 1, n) if t[i] == at]
            if not follow:
                break
            at = int(r.choice(follow))
            s[t[at]] = d[at]
        drafted.append(d)
        sampled.append(s)
    return drafted, sampled


# heads of every padding; chunks of more tokens than a pass moves (28 of 128 channels); pages that end inside a branch
@pytest.mark.parametrize("D,G,layers", [(64, 3, 2), (40, 1, 1), (128, 2, 3), (256, 1, 2)])
@pytest.mark.parametrize("counts,kinds,depth", [([1], ("tree",), 0), ([9, 0, 1, 24], ("tree",), 6), ([64, 130], ("comb", "chain"), 200), ([130], ("comb",), 200), ([40, 33], ("star", "tree"), 5), ([20, 30], ("forest",), 9)])
def test_accept_drafts(g, D, G, layers, counts, kinds, depth):
    r = np.random.default_rng(D + sum(counts))
    trees, lens, cu = _batch(r, counts, kinds)
    drafted, sampled = _tokens(r, trees, depth)
    per = -(-max(lens) // 64)
    pages = len(counts) * per + 1
    table = r.permutation(pages)[:len(counts) * per].reshape(len(counts), per).astype(np.int32)
    caches = [r.integers(0, 256, (pages, G, 72 * ref.padded(D))).astype(np.uint8) for _ in range(layers)]
    i32 = lambda x: dev(np.concatenate(x).astype(np.int32))  # noqa: E731
    n = max(counts)
    on_gpu = [dev(c) for c in caches]
    got = [host(x) for x in g.accept_drafts(i32(drafted), i32(sampled), i32(trees), dev(np.array(lens, np.int32)), cu_q=dev(cu), max_q=n, caches=on_gpu, block_table=dev(table))]
    pairs = []
    for b, t in enumerate(trees):
        kept, answer = drafts.accepted(t, drafted[b], sampled[b])
        before = lens[b] - len(t)
        assert got[0][b].tolist() == kept + [-1] * (n - len(kept)) and got[1][b] == len(kept) and got[2][b] == answer and got[3][b] == before + len(kept)
        pairs += [(drafts.slots(table[b], before + j), drafts.slots(table[b], before + i)) for i, j in enumerate(kept)]
    assert depth == 0 or max(got[1]) > 1
    for c, now in zip(caches, on_gpu):
        assert np.array_equal(host(now), drafts.moved(c, D, pairs))
    # without caches, and with as many tokens each
    again = g.accept_drafts(i32(drafted), i32(sampled), i32(trees), dev(np.array(lens, np.int32)), cu_q=dev(cu), max_q=n)
    assert all(np.array_equal(host(a), b) for a, b in zip(again, got))


# heads of one layer for more than one workgroup
@pytest.mark.parametrize("D,G", [(256, 17), (64, 60), (128, 29)])
def test_accept_drafts_of_many_heads(g, D, G):
    test_accept_drafts(g, D, G, 2, [9, 70], ("tree", "comb"), 200)


def test_accept_drafts_where_places_are_missing(g):
    """No page in the table, a page that the cache has not, a history that is shorter than the new tokens, a drawn token that is none, more nodes than max_q"""
    r = np.random.default_rng(8)
    D, G = 64, 2
    cache = r.integers(0, 256, (4, G, 72 * 64)).astype(np.uint8)
    table = np.array([[0, -1], [1, 99], [2, 3], [3, 2], [3, 0]], np.int32)
    # four stars, of which node 5 (or 3) is the first with the drawn token, and a chain with nothing drawn behind its third node
    parents = np.r_[np.zeros(24), -1, 0, 1, 2, 3, 4].astype(np.int32)
    drafted = np.array([[1, 2, -1, 4, 4, 5]] * 2 + [[1, 2, -1, 5, 5, 5]] * 2 + [[9, 5, 6, 7, 8, 4]], np.int32).ravel()
    sampled = np.array([[5, 7, 7, 7, 7, 8]] * 2 + [[5, 7, 7, 8, 7, 7]] * 2 + [[5, 6, -1, 8, 4, 3]], np.int32).ravel()
    lens = np.array([66, 67, 4, 40, 20], np.int32)
    now = dev(cache)
    got = [host(x) for x in g.accept_drafts(dev(drafted), dev(sampled), dev(parents), dev(lens), caches=[now], block_table=dev(table))]
    assert got[1].tolist() == [2, 2, 2, 2, 3] and got[2].tolist() == [8, 8, 8, 8, -1] and got[3].tolist() == [62, 63, 0, 36, 17]
    assert got[0].tolist() == [[0, k, -1, -1, -1, -1] for k in (5, 5, 3, 3)] + [[0, 1, 2, -1, -1, -1]]
    assert np.array_equal(host(now), drafts.moved(cache, D, [(3 * 64 + 37, 3 * 64 + 35)]))
    cut = [torch.full(s, 77, dtype=torch.int32, device="cuda") for s in ((5, 4), (5,), (5,), (5,))]
    cu = dev(np.array([0, 6, 12, 18, 24, 30], np.int32))
    g.calls.gpusq_accept_drafts(dev(drafted), dev(sampled), dev(parents), dev(lens), cu, None, None, 0, *cut, 30, 5, 4, 0, 0, 0, 0)
    assert host(cut[1]).tolist() == [1, 1, 2, 2, 3] and host(cut[2]).tolist() == [5, 5, 8, 8, -1] and host(cut[3]).tolist() == [61, 62, 0, 36, 17]


def test_many_caches(g):
    """More layers than one launch takes"""
    r = np.random.default_rng(5)
    t = np.array([-1, 0, 0, 2], np.int32)
    drafted, sampled = np.array([0, 1, 2, 3], np.int32), np.array([2, 0, 3, 9], np.int32)
    caches = [r.integers(0, 256, (2, 1, 72 * 64)).astype(np.uint8) for _ in range(131)]
    now = [dev(c) for c in caches]
    got = g.accept_drafts(dev(drafted), dev(sampled), dev(t), dev(np.array([66], np.int32)), caches=now, block_table=dev(np.array([[1, 0]], np.int32)))
    assert host(got[0])[0].tolist() == [0, 2, 3, -1]
    for c, x in zip(caches, now):
        assert np.array_equal(host(x), drafts.moved(c, 64, [(0 * 64 + 0, 64 + 63), (0 * 64 + 1, 0 * 64 + 0)]))


def test_refusals(g):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    t, lens, table = i32(8), i32(2), i32(2, 3)
    cache = g.kv4_cache(4, 2, 64)
    for call in (lambda: g.draft_tree(t.long(), lens, table), lambda: g.draft_tree(t, lens, table[:1]), lambda: g.draft_tree(t, lens, table, cu_q=i32(2)), lambda: g.draft_tree(t.cpu(), lens, table),
                 lambda: g.accept_drafts(t, t[:7], t, lens), lambda: g.accept_drafts(t, t, t, lens, caches=[cache]), lambda: g.accept_drafts(t, t, t, lens, caches=[cache, cache[:3]], block_table=table),
                 lambda: g.accept_drafts(t, t, t, lens, caches=[cache[:, :, :4600]], block_table=table), lambda: g.accept_drafts(t, t, t, lens, caches=[cache.cpu()], block_table=table)):
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: g.draft_tree(i32(9), lens, table), g.ERR_SHAPE), (lambda: g.draft_tree(t, lens, table, max_q=9), g.ERR_SHAPE), (lambda: g.draft_tree(t, lens, table, max_q=0), g.ERR_SHAPE),
                         (lambda: g.draft_tree(i32(1026), lens, table), g.ERR_UNSUPPORTED), (lambda: g.accept_drafts(t, t, t, lens, caches=[cache, cache], block_table=table), g.ERR_UNSUPPORTED)):
        with pytest.raises(g.GpusqError) as e:
            call()
        assert e.value.status == status
