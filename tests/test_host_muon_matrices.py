"""The list of matrices of a step: triples of integers, or refused. No library call is reached."""
import types

import numpy as np
import pytest


@pytest.mark.parametrize("bad", [[(0, 5), (5, 5), (10, 5)], [0, 5, 5], [(0, 5, 5, 1)], [[(0, 5, 5)]], [(0.5, 5, 5)], np.zeros((2, 3))])
def test_what_is_no_list_of_triples_is_refused(bad):
    import torch
    import paper_2304_14698_amd as xrl
    me = types.SimpleNamespace(torch=torch, lib=None, handle=None)
    with pytest.raises(ValueError, match="matrices"):
        xrl.Encoder.muon_step(me, torch.zeros(100), torch.zeros(100), torch.zeros(100), bad, lr=0.1)
