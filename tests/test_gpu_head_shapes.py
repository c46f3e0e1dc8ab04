"""Shapes that the output head's binding refuses though their number of elements fits."""
import pytest
import torch

import paper_2005_04680_amd as pk
from gpu_util import DEV, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


@pytest.mark.parametrize("shape", [(4, 2), (1, 8), (8, 1), (2, 3), (9,), (2, 4, 2)])
def test_teacher_logits_have_the_shape_of_their_ids(shape):
    """(A flat list of them is taken row by row.)"""
    logits = torch.zeros(2, 9, device=DEV)
    ids = torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4)
    t = torch.arange(8, dtype=torch.float32, device=DEV)
    loss, flat = torch.zeros(2, device=DEV), torch.ones(2, device=DEV)
    ws = torch.empty(1 << 12, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        pk.embbag_distill(logits, ids, torch.zeros(shape, device=DEV), 1.0, loss, ws)
    pk.check(pk.embbag_distill(logits, ids, t.view(2, 4), 1.0, loss, ws))
    pk.check(pk.embbag_distill(logits, ids, t, 1.0, flat, ws))
    assert torch.equal(loss, flat) and (loss > 0).all()
