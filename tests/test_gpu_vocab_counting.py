"""The example's model, taught to count, counts: the ids it draws are those it was taught, by its logits and through the sampling call."""
import pytest
import torch

from vocab_util import DEV

pytestmark = pytest.mark.gpu


def test_the_example_counts():
    from paper_2512_00719_amd import vocab_step
    V = 300
    model = vocab_step.TiedModel(V, 128, seed=1)
    ids = torch.arange(V, device=DEV, dtype=torch.int32)
    targets = (ids + 1) % V
    for _ in range(200):
        loss = model.train_step(ids, targets, rate=1.0)
        if float(loss) < 0.05:
            break
    assert float(loss) < 0.05
    assert torch.equal(model.logits(ids).argmax(1).to(torch.int32), targets)
    first = torch.tensor([0, 41, 150, 297], device=DEV, dtype=torch.int32)
    drawn = vocab_step.decode(model, first, 5)
    assert float((drawn == (first[:, None] + torch.arange(1, 6, device=DEV)) % V).float().mean()) >= 0.9
