"""Arguments of the link prediction that are refused instead of being without effect."""
import numpy as np
import pytest

from paper_2005_13789_amd import linkpred


@pytest.mark.parametrize("mode", ["sync", "walks", "async"])
@pytest.mark.parametrize("args,kw", [(["--optimizer", "muon"], dict(optimizer="muon")), (["--entropy-weight", "0.1"], dict(entropy_weight=0.1))])
def test_options_of_the_full_softmax_are_refused_elsewhere(mode, args, kw):
    with pytest.raises(SystemExit):
        linkpred.main(["nowhere.txt", "--mode", mode, *args])
    with pytest.raises(ValueError, match="softmax"):
        linkpred.train(np.zeros((1, 2), dtype=np.int64), 2, mode=mode, **kw)


def test_hits_of_no_edges_are_refused():
    class Nothing:
        class vertex:
            device = "cpu"
        num_nodes, dim = 4, 4
    with pytest.raises(ValueError, match="edge"):
        linkpred.hits(Nothing, np.zeros((0, 2)))
