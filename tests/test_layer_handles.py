"""Layers as handles: what they keep for their calls does not stand in the way of copying or storing them (host logic)."""
import copy
import pickle

import pytest
import torch

from paper_2410_09615_amd import binding as B


def _block():
    layer = B.SlimBlockFp8Weight(64, 128, torch.arange(64 * 128).to(torch.uint8), torch.ones(1, 1))
    struct = B.slim_block_fp8_layer(64, 128, layer.codes.data_ptr(), layer.scales.data_ptr())
    layer.__dict__["_ref"] = object.__new__(B._LayerRef)                # as a product leaves it (c_ref itself asks for device tensors)
    layer.__dict__["_ref"].layer = struct
    return layer


def _packed():
    s = B.slim_packed_sizes(64, 128, 0)
    layer = B.SlimLayer(64, 128, 0, 0, torch.arange(s["qvals"]).to(torch.uint8), torch.zeros(s["meta"], dtype=torch.uint8), torch.ones(64), None, None)
    layer.c_ref()
    return layer


@pytest.mark.parametrize("make", [_block, _packed])
@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda t: pickle.loads(pickle.dumps(t))])
def test_a_layer_that_has_been_used_can_be_copied(make, how):
    layer = make()
    assert "_ref" in layer.__dict__
    other = how(layer)
    assert "_ref" not in other.__dict__ and "_ref" in layer.__dict__
    for name, value in layer.__dict__.items():
        if name != "_ref":
            assert torch.equal(getattr(other, name), value) if isinstance(value, torch.Tensor) else getattr(other, name) == value
