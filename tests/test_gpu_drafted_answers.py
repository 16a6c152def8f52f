"""The operators of an answer with drafted tokens together, as pipeline.DraftedAnswers runs them: against the same layers answering one token a step, each
operator's definition, and replayed from a graph."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D, H, KV, HD, HIDDEN, B, S, SD, GROUP, LAYERS, V, PROMPT, MOST = 256, 8, 2, 64, 512, 3, 40, 128, 64, 2, 1000, 61, 3
PAGES = 2 + B * MOST
F32 = np.float32


def _rms(x):
    y = x.float()
    return (y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6)).half()


class Model:
    def __init__(self):
        from paper_2305_10727_amd.pipeline import DecoderLayer, DraftedAnswers
        r = np.random.default_rng(3)
        self.layers = []
        states, bias = dev(r.standard_normal((B, S, SD)).astype(np.float16)), dev(np.zeros(2 * KV * HD, F32))
        for _ in range(LAYERS):
            layer = DecoderLayer(D, H, KV, HD, HIDDEN, B, S, SD, PAGES, group=GROUP)
            layer.prepare_weights({n: dev((r.standard_normal(shape) * 0.06).astype(F32)) for n, shape in layer.widths.items()},
                                  dev((r.standard_normal((2 * KV * HD, SD)) * 0.06).astype(F32)))
            layer.see(states, bias)
            self.layers.append(layer)
        self.answers = DraftedAnswers(self.layers, V)
        self.answers.prepare_weights(dev((r.standard_normal((V, D)) * 0.06).astype(F32)))
        self.embedding = dev(r.standard_normal((V, D)).astype(np.float16))
        a = np.arange(64 * MOST)[:, None] * 10000.0 ** (-np.arange(0, HD, 2) / HD)
        self.rope = dev(np.cos(a).astype(F32)), dev(np.sin(a).astype(F32))
        self.norms = [(_rms, _rms, _rms)] * LAYERS
        self.table = dev(r.permutation(PAGES)[:B * MOST].reshape(B, MOST).astype(np.int32))
        self.prompt = r.integers(0, V, (B, PROMPT)).astype(np.int32)

    def embed(self, tokens):
        return self.embedding.index_select(0, tokens)

    def read(self):
        """The prompt but its last token, into fresh caches"""
        t = np.arange(PROMPT - 1, dtype=np.int32)
        table = host(self.table)
        slots = np.concatenate([table[b, t // 64] * 64 + t % 64 for b in range(B)]).astype(np.int32)
        for layer in self.layers:
            layer.cache.zero_()
        x = self.embed(dev(np.ascontiguousarray(self.prompt[:, :-1]).reshape(-1)))
        for layer, norms in zip(self.layers, self.norms):
            x = layer.forward(x, norms, self.rope, dev(np.tile(t, B)), dev(slots), self.table, dev(np.full(B, PROMPT - 1, np.int32)))
        return self.prompt[:, -1].copy(), np.full(B, PROMPT - 1, np.int32)

    def arguments(self, drafted, parents, lens, random=None, **kw):
        n = drafted.shape[1]
        random = np.full(B * n, 0.5, F32) if random is None else random
        args = (dev(np.ascontiguousarray(drafted, np.int32).reshape(-1)), dev(np.ascontiguousarray(parents, np.int32).reshape(-1)), dev(random), self.embed, self.norms, _rms, self.rope, self.table,
                dev((lens + n).astype(np.int32)))
        return args, {k: dev(v) for k, v in kw.items()}


@pytest.fixture(scope="module")
def model(g):
    return Model()


def _greedy(n):
    return dict(temperature=np.zeros(B * n, F32))


def _one_at_a_time(model, steps):
    """-> answers [steps, B], logits [steps, B, V]"""
    last, lens = model.read()
    answers, logits = [], []
    for _ in range(steps):
        args, kw = model.arguments(last[:, None], np.full((B, 1), -1), lens, **_greedy(1))
        path, accepted, answer, new = (host(t) for t in model.answers.step(*args, **kw))
        assert (path == 0).all() and (accepted == 1).all() and np.array_equal(new, lens + 1)
        logits.append(host(model.answers.logits).reshape(B, V))
        assert np.array_equal(answer, logits[-1].argmax(-1))
        answers.append(answer)
        last, lens = answer, new
    return np.array(answers), np.array(logits)


# Between a token alone and one of a tree lie sums in another order and the roundings to fp16 and to 4 and 8 bits that these flip: both are within 20
# roundings to fp16 of the layer's definition for each layer (of the other test of these layers), whose flips of a code of the cache (1 / 14 of a group's
# greatest) and of the vocabulary's (1 / 254 of a token's) are of single values of many hundreds
LOGITS = 0.05


def test_drafts_of_a_tree_answer_as_single_tokens_do(model):
    """Trees with the true continuation down one branch, for some way, and other tokens beside it"""
    steps = 24
    answers, logits = _one_at_a_time(model, steps)
    r = np.random.default_rng(5)
    last, lens = model.read()
    # node numbers of the true branch within the tree, and the tree: children in front of and behind the true ones
    parents = np.array([-1, 0, 0, 1, 2, 4, 2, 4, 7, 7, 5])
    branch = [0, 2, 4, 7, 9]  # (the node behind each: the true one)
    done, most = np.zeros(B, int), 0
    for step in range(5):
        n = len(parents)
        drafted = r.integers(0, V, (B, n)).astype(np.int32)
        drafted[:, 0] = last
        right = (step + np.arange(B)) % 5  # drafts that are right, of each sequence
        for b in range(B):
            for j in range(1, right[b] + 1):
                drafted[b, branch[j]] = answers[done[b] + j - 1, b]
        args, kw = model.arguments(drafted, np.tile(parents, (B, 1)), lens, **_greedy(n))
        path, accepted, answer, new = (host(t) for t in model.answers.step(*args, **kw))
        got = host(model.answers.logits).reshape(B, n, V)
        sampled = got.argmax(-1)
        for b in range(B):
            kept, behind = drafts.accepted(parents, drafted[b], sampled[b])
            assert accepted[b] == len(kept) and path[b].tolist() == kept + [-1] * (n - len(kept)) and answer[b] == behind and new[b] == lens[b] + len(kept)
            # against single tokens, node by node of the true branch
            for j, node in enumerate(branch[:right[b] + 1]):
                alone = logits[done[b] + j, b]
                assert np.abs(got[b, node] - alone).max() <= LOGITS * np.abs(alone).max()
            best = np.sort(logits[done[b]:done[b] + right[b] + 1, b], -1)
            assert (best[:, -1] - best[:, -2] <= 2 * LOGITS * best[:, -1]).any() or len(kept) >= right[b] + 1
            most = max(most, len(kept))
        if not all(np.array_equal(answers[done[b] + accepted[b] - 1, b], answer[b]) for b in range(B)):
            break  # (two tokens closer than the tolerance: another answer from here on)
        last, lens, done = answer, new, done + accepted
    assert most == 5 or step < 4


def test_drawn_tokens_and_caches_follow_the_definitions(model):
    """With temperatures and cuts: a token behind each node from its logits, the kept branch, the caches' places in each layer"""
    r = np.random.default_rng(8)
    last, lens = model.read()
    n = 7
    parents = np.array([[-1, 0, 0, 1, 2, 2, 3], [-1, 0, 1, 2, 3, 4, 5], [-1, -1, 0, 1, 0, 7, 4]])
    table = host(model.table)
    for step in range(3):
        drafted = r.integers(0, V, (B, n)).astype(np.int32)
        drafted[:, 0] = last
        u, T = r.random(B * n).astype(F32), r.choice(np.array([0, 0.5, 1.0], F32), B * n)
        k, p = r.choice(np.array([0, 1, 40], np.int32), B * n), r.choice(np.array([1, 0.9], F32), B * n)
        args, kw = model.arguments(drafted, parents, lens, u, temperature=T, top_k=k, top_p=p)
        # a first run names what is drawn; drafts that it would keep are put in its place (they change what is behind them)
        for turn in range(3):
            before = [layer.cache.clone() for layer in model.layers]
            path, accepted, answer, new = (host(t) for t in model.answers.step(*args, **kw))
            logits = host(model.answers.logits)
            sampled = []
            for i in range(B * n):
                token, _, gap = drafts.sample(logits[i], u[i], T[i], k[i], p[i])
                if gap < 2.0 ** -26:
                    pytest.skip("a random number at a token's border")
                sampled.append(token)
            sampled = np.array(sampled).reshape(B, n)
            now = host(args[0]).reshape(B, n)
            for b in range(B):
                kept, behind = drafts.accepted(parents[b], now[b], sampled[b])
                assert accepted[b] == len(kept) and path[b].tolist() == kept + [-1] * (n - len(kept)) and answer[b] == behind and new[b] == lens[b] + len(kept)
            if turn < 2:
                for layer, c in zip(model.layers, before):
                    layer.cache.copy_(c)
                for b in range(B):
                    for i in range(1, n):
                        if 0 <= parents[b, i] < i:
                            now[b, i] = sampled[b, parents[b, i]]
                args[0].copy_(dev(now.reshape(-1)))
        assert accepted.max() > 1
        # the caches: what the layers wrote, moved.  (Written again without the last call, on the caches as they were)
        after = [host(layer.cache) for layer in model.layers]
        for layer, c in zip(model.layers, before):
            layer.cache.copy_(c)
        from paper_2305_10727_amd import gpusq as G
        tree, positions, slots = G.draft_tree(args[1], args[8], model.table)
        x = model.embed(args[0])
        for layer, norms in zip(model.layers, model.norms):
            x = layer.forward(x, norms, model.rope, positions, slots, model.table, args[8], tree=tree)
        for layer, got in zip(model.layers, after):
            pairs = [(drafts.slots(table[b], lens[b] + node), drafts.slots(table[b], lens[b] + i)) for b in range(B) for i, node in enumerate(path[b]) if node >= 0]
            assert np.array_equal(got, drafts.moved(host(layer.cache), HD, pairs))
            layer.cache.copy_(dev(got))
        last, lens = answer, new


def test_steps_from_a_graph(model):
    """Recorded once, replayed with the next drafts, lengths and random numbers: as eager steps, bit for bit, results and caches"""
    r = np.random.default_rng(13)
    last, lens = model.read()
    n = 6
    parents = np.tile(np.array([-1, 0, 1, 0, 3, 3]), (B, 1))
    drafted = r.integers(0, V, (B, n))
    args, kw = model.arguments(drafted, parents, lens, **_greedy(n))
    saved = [layer.cache.clone() for layer in model.layers]
    model.answers.capture(*args, **kw)
    for layer, c in zip(model.layers, saved):
        layer.cache.copy_(c)
    for step in range(5):
        drafted[:, 0] = last
        if step:  # the token behind node 0 is drafted, too
            drafted[:, 1] = known
        args[0].copy_(dev(drafted.astype(np.int32).reshape(-1)))
        args[2].copy_(dev(r.random(B * n).astype(F32)))
        args[8].copy_(dev((lens + n).astype(np.int32)))
        kw["temperature"].copy_(dev(np.full(B * n, [0.0, 1.0][step % 2], F32)))
        before = [layer.cache.clone() for layer in model.layers]
        got = [t.clone() for t in model.answers.replay()]
        logits, caches = model.answers.logits.clone(), [layer.cache.clone() for layer in model.layers]
        for layer, c in zip(model.layers, before):
            layer.cache.copy_(c)
        eager = model.answers.step(*args, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)) and torch.equal(logits, model.answers.logits)
        assert all(torch.equal(c, layer.cache) for c, layer in zip(caches, model.layers))
        known = r.integers(0, V, B)
        last, lens = host(got[2]), host(got[3])


def test_what_a_later_call_would_refuse_is_not_in_the_caches(model):
    last, lens = model.read()
    n = 2
    args, kw = model.arguments(np.repeat(last[:, None], n, 1), np.tile([-1, 0], (B, 1)), lens, temperature=np.ones(B * n, F32), top_k=np.ones(B * n, np.int32))
    before = [layer.cache.clone() for layer in model.layers]
    for at, bad in ((0, args[0][:4].contiguous()), (0, args[0].long()), (1, args[1][:5].contiguous()), (2, None), (2, args[2].double()), (4, model.norms[:1]), (7, model.table[:2].contiguous()),
                    (7, model.table.long()), (8, args[8][:1].contiguous()), (8, args[8].cpu())):
        with pytest.raises(ValueError):
            model.answers.step(*args[:at], bad, *args[at + 1:], **kw)
    for bad in (dict(temperature=kw["temperature"][:1]), dict(top_k=kw["temperature"]), dict(top_p=kw["top_k"]), dict(min_p=kw["temperature"].half()), dict(state_lens=args[8].long()),
                dict(head_weights=[(None, None)])):
        with pytest.raises(ValueError):
            model.answers.step(*args, **{**kw, **bad})
    assert all(torch.equal(c, layer.cache) for c, layer in zip(before, model.layers))
    model.answers.step(*args, **kw)
    assert not any(torch.equal(c, layer.cache) for c, layer in zip(before, model.layers))


def test_layers_that_do_not_belong_together(model):
    from paper_2305_10727_amd.pipeline import DecoderLayer, DraftedAnswers
    other = DecoderLayer(D, H, KV, HD, HIDDEN, B, S, SD, PAGES + 1, group=GROUP)
    for layers in ([], [model.layers[0], other], [model.layers[0]] * 2):
        with pytest.raises(ValueError):
            DraftedAnswers(layers, V)
    with pytest.raises(ValueError):
        model.answers.prepare_weights(model.embedding[:-1].contiguous())
