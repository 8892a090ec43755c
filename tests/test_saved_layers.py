"""Layers saved whole by a version without activations still load (CPU)."""
import pickle

import torch

from paper_2305_17190_amd.autograd import PAMLinear


def test_a_layer_without_its_activation():
    old = PAMLinear(3, 2)
    del old.__dict__["activation"]            # as such a version left it
    layer = pickle.loads(pickle.dumps(old))
    assert layer.activation is None and "activation" not in repr(layer)
    assert torch.equal(layer.weight, old.weight)
    assert PAMLinear(3, 2, activation="gelu").activation == "gelu"
