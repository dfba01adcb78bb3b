"""CPU: lists of gradients that hold something else than dense tensors (a parameter without a gradient has None) are refused like every call that does not fit."""
import pytest
import torch

import paper_2508_18376_amd as ds


def z(*shape):
    return torch.zeros(*shape)


SPARSE = torch.sparse_coo_tensor([[0, 2]], [1.0, 2.0], (4,))
OTHERS = {"None": None, "a number": 1.0, "a list": [1.0], "a sparse tensor": SPARSE}


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("other", OTHERS)
def test_gradients(other, first):
    grads = [OTHERS[other], z(4)] if first else [z(4), OTHERS[other]]
    for call in (ds.moe_grad_norm, lambda g: ds.moe_clip_grads(g, 1.0), lambda g: ds.moe_clip_grads(g, 1.0, out=g), lambda g: ds.moe_clip_grads(g, 1.0, out=[z(4), z(4)])):
        with pytest.raises(ds.DsmoeError, match="list of tensors") as e:
            call(grads)
        assert e.value.status == -1


@pytest.mark.parametrize("other", OTHERS)
def test_outputs(other):
    with pytest.raises(ds.DsmoeError, match="list of") as e:
        ds.moe_clip_grads([z(4), z(4)], 1.0, out=[z(4), OTHERS[other]])
    assert e.value.status == -1
