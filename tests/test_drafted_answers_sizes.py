"""Which sizes pipeline.DraftedAnswers takes, on the host: what every step would refuse behind its layers is refused here.  No kernel is launched."""
import types

import pytest

torch = pytest.importorskip("torch")


def _answers(vocabulary, D=64, layers=2):
    from paper_2305_10727_amd.pipeline import DraftedAnswers
    cache = torch.zeros((3, 2, 72 * 64), dtype=torch.uint8)
    return DraftedAnswers([types.SimpleNamespace(batch=2, D=D, cache=cache) for _ in range(layers)], vocabulary, device="cpu")


@pytest.mark.parametrize("vocabulary", [1, 2, 3, 4, 997, 32001, 50257, 2**18 - 1, 2**18])
def test_any_vocabulary_has_weights_that_the_product_takes(vocabulary):
    """Rows in fours, those behind the vocabulary's zeros"""
    a = _answers(vocabulary)
    rows = a.Wq.shape[0]
    assert rows % 4 == 0 and vocabulary <= rows < vocabulary + 4 and a.Wq.shape == (rows, 64) and a.w_scale.shape == (rows,)
    assert not a.Wq[vocabulary:].any() and not a.w_scale[vocabulary:].any()


@pytest.mark.parametrize("vocabulary,D,layers", [(0, 64, 2), (-4, 64, 2), (2**18 + 1, 64, 2), (2**18 + 4, 64, 2), (1000, 24, 2), (1000, 0, 2), (8, 132112, 1), (1000, 64, 1025)])
def test_sizes_that_a_step_would_refuse(vocabulary, D, layers):
    with pytest.raises(ValueError):
        _answers(vocabulary, D, layers)
