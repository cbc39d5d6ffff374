"""What the dropout calls make of their seed before anything is launched."""
import inspect

import pytest


def test_a_seed_is_needed_where_elements_are_drawn():
    import torch
    from paper_2506_10315_amd import ops
    x = torch.zeros(2, 3)
    for p in (1e-6, 0.1, 0.999):
        with pytest.raises(ValueError, match="without a seed"):
            ops._seed(None, 0, x, p)
        assert ops._seed(7, 2, x, p) == (7, None, 2)
    for p in (0.0, 1.0, -0.1):   # the last is the boundary's to refuse
        assert ops._seed(None, 4, x, p) == (0, None, 4)
    for call in (ops.dropout_add_layer_norm, ops.dropout_add_layer_norm_forward, ops.dropout_add_layer_norm_backward):
        assert inspect.signature(call).parameters["seed"].default is None
