"""pipeline.DraftedAnswers: vocabularies of any size, and arguments that a later call of a step would refuse: before the caches are written."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_drafted_answers import B, D, F32, LAYERS, V, Model
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PARENTS = np.array([-1, 0, 0, 1, 2])


@pytest.fixture(scope="module")
def model(g):
    return Model()


def _step_arguments(model, r):
    last, lens = model.read()
    n = len(PARENTS)
    drafted = r.integers(0, 900, (B, n)).astype(np.int32)
    drafted[:, 0] = last
    T = r.choice(np.array([0, 0.7, 1.0], F32), B * n)
    return model.arguments(drafted, np.tile(PARENTS, (B, 1)), lens, r.random(B * n).astype(F32), temperature=T, top_k=np.full(B * n, 40, np.int32), top_p=np.full(B * n, 0.9, F32),
                           min_p=np.zeros(B * n, F32)), drafted, T, lens


@pytest.mark.parametrize("vocabulary", [997, 998, 999])
def test_a_vocabulary_that_is_no_multiple_of_4(model, vocabulary):
    """Logits as a larger one's first, tokens by their definition, eagerly and from a graph"""
    from paper_2305_10727_amd.pipeline import DraftedAnswers
    r = np.random.default_rng(vocabulary)
    W = (np.random.default_rng(31).standard_normal((V, D)) * 0.06).astype(F32)
    whole, some = DraftedAnswers(model.layers, V), DraftedAnswers(model.layers, vocabulary)
    whole.prepare_weights(dev(W))
    some.prepare_weights(dev(W[:vocabulary]))
    (args, kw), drafted, T, lens = _step_arguments(model, r)
    saved = [layer.cache.clone() for layer in model.layers]

    def fresh():
        for layer, c in zip(model.layers, saved):
            layer.cache.copy_(c)

    whole.step(*args, **kw)
    logits = host(whole.logits)
    fresh()
    got = [host(t) for t in some.step(*args, **kw)]
    assert some.logits.shape == (len(drafted) * len(PARENTS), vocabulary) and np.array_equal(host(some.logits), logits[:, :vocabulary])
    u = host(args[2])
    sampled = []
    for i in range(len(u)):
        token, _, gap = drafts.sample(logits[i, :vocabulary], u[i], T[i], 40, F32(0.9))
        if gap < 2.0 ** -26:
            pytest.skip("a random number at a token's border")
        sampled.append(token)
    for b in range(B):
        kept, behind = drafts.accepted(PARENTS, drafted[b], np.array(sampled).reshape(B, -1)[b])
        assert got[0][b].tolist() == kept + [-1] * (len(PARENTS) - len(kept)) and got[1][b] == len(kept) and got[2][b] == behind and got[3][b] == lens[b] + len(kept)
    fresh()
    some.capture(*args, **kw)
    for _ in range(3):
        fresh()
        again = some.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(host(a), b) for a, b in zip(again, got)) and np.array_equal(host(some.logits), logits[:, :vocabulary])


def _apart(t):
    """The same values with others between them"""
    return torch.stack([t, t], -1)[..., 0]


def test_arguments_with_gaps_are_refused_in_front_of_the_caches(model):
    from paper_2305_10727_amd import gpusq as G
    r = np.random.default_rng(1)
    (args, kw), *_ = _step_arguments(model, r)
    before = [layer.cache.clone() for layer in model.layers]
    for at in (0, 1, 2, 7, 8):  # drafted, parents, random, the table, lengths
        with pytest.raises(ValueError):
            model.answers.step(*args[:at], _apart(args[at]), *args[at + 1:], **kw)
    for name, t in kw.items():
        with pytest.raises(ValueError):
            model.answers.step(*args, **{**kw, name: _apart(t)})
    states = torch.full((B,), 5, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        model.answers.step(*args, **kw, state_lens=_apart(states))
    assert all(torch.equal(c, layer.cache) for c, layer in zip(before, model.layers))
    # a layer by itself
    tree, positions, slots = G.draft_tree(args[1], args[8], model.table)
    x, layer = model.embed(args[0]), model.layers[0]
    call = lambda table=model.table, lens=args[8], **k: layer.forward(x, model.norms[0], model.rope, positions, slots, table, lens, **k)  # noqa: E731
    for bad in (dict(tree=_apart(tree)), dict(tree=tree, table=_apart(model.table)), dict(tree=tree, lens=_apart(args[8])), dict(tree=tree, state_lens=_apart(states)),
                dict(table=_apart(model.table)), dict(lens=_apart(args[8])), dict(state_lens=_apart(states))):
        with pytest.raises(ValueError):
            call(**bad)
    assert all(torch.equal(c, layer.cache) for c, layer in zip(before, model.layers))
    assert LAYERS == len(model.layers)
    call(tree=tree, state_lens=states)
    assert not torch.equal(before[0], layer.cache)
