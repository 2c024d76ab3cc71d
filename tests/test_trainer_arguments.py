"""Arguments of the full-softmax trainer that are refused when it is made, not in the middle of a step."""
import pytest
import torch

from paper_2005_13789_amd.fullsoftmax import SoftmaxTrainer


@pytest.mark.parametrize("kw", [dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=float("nan")), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
                                dict(weight_decay=float("inf")), dict(momentum=1 - 1e-9), dict(weight_decay=1e39)])
def test_muon_refuses_what_its_steps_would(kw):
    t = torch.zeros(5, 4)
    with pytest.raises(ValueError, match="Muon"):
        SoftmaxTrainer(t, t.clone(), 4, optimizer="muon", **kw)
