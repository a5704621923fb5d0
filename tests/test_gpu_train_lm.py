"""The example that uses the training operators with the compression step: a language model learns its synthetic language.

One token in ten is drawn at random from the vocabulary, so the best possible loss is the entropy of that mixture, and the
best token is right for 0.9 + 0.1 / vocab of the tokens."""
import math

import pytest

from paper_1903_04488_b200 import train_lm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_the_example_learns(cuda_device, state):
    vocab = 64
    report = train_lm.train(steps=120, workers=3, vocab=vocab, dim=48, layers=1, tokens=512, lr=0.3, state=state, report_every=119,
                            quiet=True)
    hit = 0.9 + 0.1 / vocab
    best = -hit * math.log(hit) - (1 - hit) * math.log(0.1 / vocab)
    (_, first, _, _), (_, last, entropy, right) = report
    assert first > math.log(vocab)                     # an untrained model is worse than guessing evenly
    # 1536 tokens: the share of right ones is within 6 standard deviations, the loss within reach of the best
    assert abs(right - hit) <= 6 * math.sqrt(hit * (1 - hit) / 1536)
    assert last <= best + 0.5 and entropy <= best + 0.5
