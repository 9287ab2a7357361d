"""Edges of the serving calls that ordinary batches do not reach."""
import pytest
import torch

from tests.test_gpu_serving_ops import DEV, context

pytestmark = pytest.mark.gpu


def test_compacting_the_pages_of_no_sequence_says_that_none_is_in_use():
    dl, ctx = context(4, 64)
    pg = dl.Pages(0, 6, 2, 16, DEV)
    live = torch.full((1,), 7, dtype=torch.int32, device=DEV)
    ctx.pages_compact(pg, [], live)
    assert live.item() == 0
    ctx.pages_compact(pg, [])
    assert ctx.device_status()[0] == 0
    ctx.close()
