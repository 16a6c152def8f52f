"""Greedy answers of drafted steps against the same layers answering one token a step, sequence by sequence: a sequence may only part from the other run where the
two best tokens are closer than the tolerance, and is left out from there on."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_drafted_answers import B, D, F32, LOGITS, Model, _greedy
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

STEPS = 6
# children in front of and behind the true ones; the node behind each of `BRANCH` is the true continuation
PARENTS, BRANCH = np.array([-1, 0, 0, 1, 2, 4, 2, 4, 7, 7, 5]), [0, 2, 4, 7, 9]


# Few tokens, so that the best one is mostly far in front: of 16 normal logits the two best are closer than 2 LOGITS of the greatest in a quarter of the positions, and
# apart by a tenth of that in nearly all
@pytest.mark.parametrize("vocabulary,seed", [(16, 0), (16, 1), (13, 2), (61, 3)])
def test_trees_answer_as_single_tokens_do(g, vocabulary, seed):
    from paper_2305_10727_amd.pipeline import DraftedAnswers
    model = Model()
    r = np.random.default_rng(seed)
    answers = DraftedAnswers(model.layers, vocabulary)
    answers.prepare_weights(dev((r.standard_normal((vocabulary, D)) * 0.06).astype(F32)))

    # one token a step
    last, lens = model.read()
    true, logits = [], []
    for _ in range(STEPS * len(BRANCH)):
        args, kw = model.arguments(last[:, None], np.full((B, 1), -1), lens, **_greedy(1))
        _, _, answer, lens = (host(t) for t in answers.step(*args, **kw))
        logits.append(host(answers.logits))
        assert np.array_equal(answer, logits[-1].argmax(-1))
        true.append(answer)
        last = answer
    true, logits = np.array(true), np.array(logits)
    best = np.sort(logits, -1)
    close = best[..., -1] - best[..., -2] <= 2 * LOGITS * np.abs(logits).max(-1)  # [position, sequence]

    last, lens = model.read()
    done, together, compared, longest = np.zeros(B, int), np.ones(B, bool), 0, 0
    n = len(PARENTS)
    for step in range(STEPS):
        drafted = r.integers(0, vocabulary, (B, n)).astype(np.int32)
        drafted[:, 0] = last
        right = (step + np.arange(B)) % len(BRANCH)  # drafts that are right, of each sequence
        for b in range(B):
            for j in range(1, right[b] + 1):
                drafted[b, BRANCH[j]] = true[done[b] + j - 1, b]
            for node in (1, 3):  # node 1, a child of node 0 in front of the true one, is not the true token
                if together[b] and drafted[b, node] == true[done[b], b]:
                    drafted[b, node] = (drafted[b, node] + 1) % vocabulary
        args, kw = model.arguments(drafted, np.tile(PARENTS, (B, 1)), lens, **_greedy(n))
        path, accepted, answer, new = (host(t) for t in answers.step(*args, **kw))
        got = host(answers.logits).reshape(B, n, vocabulary)
        for b in range(B):
            kept, behind = drafts.accepted(PARENTS, drafted[b], got[b].argmax(-1))
            assert accepted[b] == len(kept) and path[b].tolist() == kept + [-1] * (n - len(kept)) and answer[b] == behind and new[b] == lens[b] + len(kept)
            if not together[b]:
                continue
            # the true branch's nodes, each as that token alone
            for j, node in enumerate(BRANCH[:right[b] + 1]):
                alone = logits[done[b] + j, b]
                assert np.abs(got[b, node] - alone).max() <= LOGITS * np.abs(alone).max(), (step, b, node)
                if got[b, node].argmax() != alone.argmax():
                    assert close[done[b] + j, b], (step, b, node)
            # the kept tokens and the answer, each as the other run's; the first that is not may only be where two are close
            tokens = [int(drafted[b, i]) for i in kept[1:]] + [int(answer[b])]
            for j, token in enumerate(tokens):
                if token != true[done[b] + j, b]:
                    assert close[done[b] + j, b], (step, b, j)
                    together[b] = False
                    break
                compared += 1
            if together[b]:
                # (of two children with the same draft the one in front is kept, here one that nothing true follows)
                twice = any(drafted[b, other] == drafted[b, node] for other, node in ((1, 2), (5, 7), (8, 9)) if node in BRANCH[:right[b] + 1])
                assert len(kept) >= right[b] + 1 or twice
                longest = max(longest, len(kept))
        last, lens, done = answer, new, done + accepted
    assert longest == len(BRANCH) and compared >= STEPS * B, (longest, compared, together)
