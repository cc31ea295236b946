"""The rank rule in the training example: the matrix it is asked about, and what it decides over a short run."""
import pytest
import torch

from paper_2511_10333_amd import train_block as tb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden,ff,sequence", [(256, 512, 128), (192, 640, 32)])
def test_the_rule_is_asked_about_the_smallest_compressed_matrix(monkeypatch, hidden, ff, sequence):
    """The smallest by elements that is compressed at every rank; and the run does get past the warm-up."""
    asked, ranks = [], []
    rule = tb.select_rank
    monkeypatch.setattr(tb, "select_rank", lambda state, h, n, prm: asked.append((prm.m, prm.n)) or rule(state, h, n, prm))
    losses = tb.train(layers=2, hidden=hidden, ff=ff, tokens=512, sequence=sequence, steps=30, window=5, dtype=torch.float32,
                      report=lambda d: ranks.append(d["rank"]))
    assert asked == 6 * [(ff, hidden)]
    assert any(r > 0 for r in ranks) and all(r == 0 or r in tb.RANKS for r in ranks)
    assert all(l == l for l in losses) and sum(losses[-5:]) < 0.8 * sum(losses[:5])
