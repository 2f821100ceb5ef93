"""Places of a batch's rows, until they are given or assigned."""
import pytest
import torch

import paper_2605_12471_amd as kv

pytestmark = pytest.mark.gpu


def test_places_of_a_batch_that_nobody_gave():
    with kv.KvFoldPagedCache(1, 8, 2, 128, 16, 4) as cache:
        batch = kv.KvFoldBatch(cache, torch.zeros((2, 2), dtype=torch.int32, device="cuda"), 5, 4, 20)
        assert (batch.slots == -1).all()
