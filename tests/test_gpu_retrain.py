"""The prune-retrain loop through the public calls: the pruned layer learns, and one step's gradients are right."""
import pytest
import torch

from paper_1911_08020_gb300 import darb, retrain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("states", ["f32", "e4m3"])
def test_a_pruned_layer_learns(states):
    before, after = retrain.retrain(steps=120, vocab=300, features=64, tokens=256, states=states)
    assert before > 300 > after   # guessing evenly has a perplexity of the vocabulary's size: worse before, better after


def test_states_in_8_bits_learn_as_well():
    full = retrain.retrain(steps=120, vocab=300, features=64, tokens=256, states="f32")[1]
    assert retrain.retrain(steps=120, vocab=300, features=64, tokens=256, states="e4m3")[1] < 1.1 * full


def test_the_encoding_follows_the_weights():
    head = retrain.Head(100, 32, 4)
    try:
        h, words = retrain.data(64, 100, 32, 0)
        head.train(h, words)
        fresh = darb.darb_encode(head.W.bfloat16(), darb.darb_export(head.handle)[3])
        for a, b in zip(darb.darb_export(head.handle), darb.darb_export(fresh)):
            assert (a == b).all()
        darb.darb_destroy(fresh)
        best = head.score(h, words, 3)
        logits = head.forward(h)[2]
        assert torch.equal(best.top_index[:, 0].long(), logits.argmax(dim=0))
    finally:
        head.close()
