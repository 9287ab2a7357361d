"""What the binding of the serving calls refuses before a kernel sees it (no GPU needed: tensors of the CPU stand in for
those of device -1)."""
import pytest
import torch

from paper_2412_00876_b200 import binding as dl


def rows(t, what="k"):
    return dl._rows(t, torch.bfloat16, tuple(t.shape), what, -1)


@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_rows_that_lie_over_one_another_are_refused(what):
    one = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=what):
        rows(one.expand(1000, 2, 64), what)                       # one row of 256 bytes, not a thousand
    flat = torch.zeros(4096, dtype=torch.bfloat16)
    for step in (8, 64, 120):
        with pytest.raises(ValueError, match=what):
            rows(flat.as_strided((10, 2, 64), (step, 64, 1)), what)


def test_rows_that_do_not_are_taken_with_their_stride():
    flat = torch.zeros(8192, dtype=torch.bfloat16)
    for step in (128, 136, 400):
        assert rows(flat.as_strided((10, 2, 64), (step, 64, 1))) == (flat.data_ptr(), step)
    assert rows(flat.as_strided((1, 2, 64), (0, 64, 1))) == (flat.data_ptr(), 128)          # one row has no next
    assert rows(flat[:0].view(0, 2, 64))[1] in (0, 128)
    with pytest.raises(ValueError, match="dense heads"):
        rows(flat.as_strided((10, 2, 64), (256, 128, 1)))
